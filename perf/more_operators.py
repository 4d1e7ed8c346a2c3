"""Operators between a projection and a cache in pages of 8 bits: rotary positions, rows quantised as they are written and
read back, and attention over such pages.

    rope          rotary positions of a step's q and k rows, or of a dense prompt's; half and interleaved layouts, part of the
                  head, frequencies scaled for long contexts; both directions
    qpage_store   new K and V rows to pages that hold e4m3 values with one power-of-two scale for 16 tokens of a head
    qpage_load    a sequence's rows out of those pages, dense, in fp16
    qpage_attn    attention of each request's new tokens (one to thousands) over those pages, with row statistics

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
BLOCK = 16                    # tokens that share a scale
MOST = 61440.0                # of a value in size: the largest number that fp16 and 8 bits with a scale of 2^8 both have


def _rope(name, T, Hq=32, Hkv=8, R=0, longest=0, rot=D, style=1, factor=1.0, trained=0, back=False, B=1):
    """R requests of a packed batch (R > 0), or B dense prompts."""
    return dict(name=name, op="rope", T=T, Hq=Hq, Hkv=Hkv, R=R, longest=longest, rot=rot, style=style, factor=factor, trained=trained, back=back, B=B)


def _attn(name, R, T, longest, Hq=32, Hkv=8, page=64, window=0, sinks=0, kind="chunk", stats=False):
    return dict(name=name, op="attn", R=R, T=T, longest=longest, Hq=Hq, Hkv=Hkv, page=page, window=window, sinks=sinks, kind=kind, stats=stats)


def listed():
    return [
        # q and k of a decode step of 64 requests, contexts up to 131072 with frequencies scaled by turns
        _rope("rope_64", 64, R=64, longest=131072, factor=8.0, trained=8192),
        # chunks of several prompts out of a fused projection
        _rope("rope_32k", 32768, R=16, longest=65536),
        # keys of two dense prompts of odd length turned back before they are encoded: interleaved, half of the head
        _rope("rope_back_4099", 4099, Hq=0, rot=64, style=0, back=True, B=2),
        # a decode step's rows into the pages of 64 requests, and those pages read back
        dict(name="store_64", op="store", R=64, T=64, Hkv=8, page=16),
        # the rows of a long prompt's chunk, beginning inside a block, and read back
        dict(name="store_32k", op="store", R=1, T=32768, Hkv=8, page=64),
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
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "rope", "store", "store", "load", "attn", "attn", "attn", "attn"])
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (32, 32), (16, 8), (28, 7)])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "rope":
        rot, style, back = rng.choice([16, 32, 64, 96, 128, 128, 128]), rng.randint(0, 1), rng.random() < 0.3
        factor, trained = rng.choice([(1.0, 0), (4.0, 0), (8.0, 8192), (32.0, 4096)])
        if rng.random() < 0.6:
            R = _log_uniform(rng, 1, 512)
            case = _rope("", _log_uniform(rng, R, 32768 * 40 // (Hq + Hkv)), Hq, Hkv, R, _log_uniform(rng, 64, 131072), rot, style, factor, trained, back)
        else:
            Hq, B = rng.choice([0, Hq]), _log_uniform(rng, 1, 8)
            case = _rope("", _log_uniform(rng, 1, 32768 * 40 // ((Hq + Hkv) * B)), Hq, Hkv, 0, 0, rot, style, factor, trained, back, B)
        del case["name"]
        return case
    if op == "store":
        R = _log_uniform(rng, 1, 256)
        return dict(op=op, R=R, T=_log_uniform(rng, R, 32768 * 8 // Hkv), Hkv=Hkv, page=page)
    if op == "load":
        R = _log_uniform(rng, 1, 8)
        return dict(op=op, R=R, N=_log_uniform(rng, 1, 32768 * 32 // (R * Hkv)), Hkv=Hkv, page=page)
    window, sinks = (0, 0) if rng.random() < 0.6 else (_log_uniform(rng, 1, 4096), rng.choice([0, 1, 4, 37]))
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


def _keys(gen, *shape):
    """Rows of keys as they come: four channels ten times the others."""
    k = torch.randn(shape, dtype=torch.float16, device="cuda", generator=gen)
    k[..., 5::32] *= 10
    return k


def _values(gen, *shape):
    return torch.randn(shape, dtype=torch.float16, device="cuda", generator=gen)


def _pool(gen, make, n_pages, Hkv, page):
    """Pages of 8 bits, [n_pages, Hkv, page, D] and their scales [n_pages, Hkv, page / 16], full of such rows."""
    pages = torch.empty((n_pages, Hkv, page, D), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((n_pages, Hkv, page // BLOCK), device="cuda")
    step = max(1, (1 << 26) // (Hkv * page * D))
    for a in range(0, n_pages, step):
        x = make(gen, min(step, n_pages - a), Hkv, page // BLOCK, BLOCK, D).float()
        s = _scale_for(x.abs().amax((-1, -2)))
        pages[a:a + step] = (x / s[..., None, None]).view(-1, Hkv, page, D).to(torch.float8_e4m3fn)
        scales[a:a + step] = s
    return pages, scales


def _pools(s, gen, n_pages):
    for name, make in (("k", _keys), ("v", _values)):
        s[name + "_pages"], s[name + "_scales"] = _pool(gen, make, n_pages, s["Hkv"], s["page"])


def _scattered(gen, counts, n_pages):
    """int32 [R, most] page numbers, no page twice, -1 behind a request's last one."""
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    most = max(max(counts), 1)
    first = _ints([sum(counts[:r]) for r in range(len(counts))], torch.int64)
    at = torch.arange(most, device="cuda")
    held = at < _ints(counts, torch.int64)[:, None]
    return torch.where(held, order[(first[:, None] + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, s = case["op"], dict(case)
    Hkv = case["Hkv"]
    if op == "rope":
        T, Hq, B = case["T"], case["Hq"], case["B"]
        if case["R"]:                                            # rows as a fused projection leaves them: token, then Q, K and V heads
            qkv = _values(gen, T, Hq + 2 * Hkv, D)
            s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
            ctx, new = _lengths(case)
            s["ctx"], s["q_start"] = _ints(ctx), _ints([sum(new[:r]) for r in range(len(new) + 1)])
        else:                                                    # dense, as prompt attention and anchor selection have it
            s["q"] = _values(gen, B, Hq, T, D) if Hq else None
            s["k"] = _keys(gen, B, Hkv, T, D)
        return s
    page = case["page"]
    if op == "store":
        R, T = case["R"], case["T"]
        rng = random.Random("%(R)d %(T)d" % case)
        held = [rng.randint(1, page) for _ in range(R)]          # rows in the page that a request goes on in
        share = [rng.random() + 0.1 for _ in range(R)]
        new = [1 + int((T - R) * w / sum(share)) for w in share]
        new[0] += T - sum(new)
        slots, n_pages = [], sum(-(-(h % page + n) // page) for h, n in zip(held, new))
        order = torch.randperm(n_pages, device="cuda", generator=gen)
        at = 0
        for h, n in zip(held, new):
            pos = torch.arange(h % page, h % page + n, device="cuda")
            slots.append(order[at + pos // page] * page + pos % page)
            at += -(-(h % page + n) // page)
        s["slot"] = torch.cat(slots).to(torch.int32)
        _pools(s, gen, n_pages)
        qkv = _values(gen, T, 6 * Hkv, D)                        # a few tokens stand out: their blocks' scales grow
        qkv *= torch.where(torch.rand((T, 1, 1), device="cuda", generator=gen) < 0.05, 8.0, 1.0).half()
        s["k"], s["v"] = qkv[:, 4 * Hkv:5 * Hkv], qkv[:, 5 * Hkv:]
        s["table"], s["N"] = order[None].to(torch.int32).contiguous(), n_pages * page
        return s
    if op == "load":
        R, N = case["R"], case["N"]
        lens = [N] + [max(1, N - 37 * r) for r in range(1, R)]
        counts = [-(-n // page) for n in lens]
        n_pages = sum(counts) + 8
        s["table"] = _scattered(gen, counts, n_pages)
        s["ctx"] = _ints(lens)
        _pools(s, gen, n_pages)
        s["k_out"], s["v_out"] = (torch.zeros((R, Hkv, N, D), dtype=torch.float16, device="cuda") for _ in "kv")
        return s
    ctx, new = _lengths(case)
    counts = [-(-c // page) for c in ctx]
    n_pages = sum(counts) + 8
    s["table"] = _scattered(gen, counts, n_pages)
    _pools(s, gen, n_pages)
    s["ctx"], s["q_start"] = _ints(ctx), _ints([sum(new[:r]) for r in range(len(new) + 1)])
    s["most_new"], s["most_ctx"] = max(new), max(ctx)            # a server knows its lengths
    s["q"] = _values(gen, case["T"], case["Hq"] + 2 * Hkv, D)[:, :case["Hq"]]
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_freqs(rot, factor, trained, base=10000.0, slow=1.0, fast=4.0):
    """Radians per position of each pair: all through `factor`, or, with a trained length, only those that turn less than `fast`
    times within it (wholly from `slow` times down)."""
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if not trained:
        return f / factor
    w = ((trained * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
    return f * (w + (1 - w) / factor)


def _plain_rope(s):
    rot, T = s["rot"], s["T"]
    f = _plain_freqs(rot, s["factor"], s["trained"])
    t = torch.arange(T, device="cuda")
    if s["R"]:
        start, ctx = s["q_start"].long(), s["ctx"].long()
        r = torch.searchsorted(start[1:].contiguous(), t, right=True)
        t = ctx[r] - start[r + 1] + t
    angle = t.double()[:, None] * f                              # 64 bits: far positions turn thousands of times
    cos, sin = angle.cos().float(), angle.sin().float() * (-1 if s["back"] else 1)
    if s["R"]:
        cos, sin = cos[:, None], sin[:, None]                    # [T, 1, pairs] beside [T, H, D]; dense: [T, pairs] beside [B, H, T, D]
    out = {}
    for name in ("q", "k"):
        x = s[name]
        if x is None:
            continue
        x = x.float()
        y = x.clone()
        a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if s["style"] else (x[..., :rot:2], x[..., 1:rot:2])
        u, v = a * cos - b * sin, b * cos + a * sin
        if s["style"]:
            y[..., :rot // 2], y[..., rot // 2:rot] = u, v
        else:
            y[..., :rot:2], y[..., 1:rot:2] = u, v
        out[name] = y.half()
    return out


def _scale_for(amax):
    """The least power of two from 2^-32 to 2^8 through which amax is at most 448."""
    e = torch.frexp(amax.clamp(min=1e-30)).exponent - 9          # amax < 2^(e + 9)
    s = torch.ldexp(torch.ones_like(amax), e)
    return torch.where(amax > 448 * s, 2 * s, s).clamp(2.0 ** -32, 2.0 ** 8)


def _dense(pages, scales, ids, off):
    """Values [.., Hkv, D] in 32 bits of pages `ids` at tokens `off`."""
    return pages.view(torch.uint8)[ids, :, off].view(torch.float8_e4m3fn).float() * scales[ids, :, off // BLOCK][..., None]


def _plain_store(s):
    page, Hkv = s["page"], s["Hkv"]
    slot = s["slot"].long()
    block = slot // BLOCK
    n_blocks = s["k_scales"].shape[0] * (page // BLOCK)
    touched, fresh = (torch.zeros(n_blocks, dtype=torch.bool, device="cuda") for _ in range(2))
    touched[block] = True
    fresh[block[slot % BLOCK == 0]] = True                       # a block that begins anew: nothing in it counts
    for name in "kv":
        pages, scales, x = s[name + "_pages"], s[name + "_scales"], s[name].float().clamp(-MOST, MOST)
        top = torch.zeros((n_blocks, Hkv), device="cuda").index_reduce_(0, block, x.abs().amax(-1), "amax")
        need = _scale_for(top).view(-1, page // BLOCK, Hkv).transpose(1, 2)
        is_fresh, is_touched = (b.view(-1, 1, page // BLOCK) for b in (fresh, touched))
        grown = torch.where(is_touched, torch.where(is_fresh, need, torch.maximum(need, scales)), scales)
        ratio = torch.where(is_fresh, 1.0, scales / grown)
        held = pages.view(-1, Hkv, page // BLOCK, BLOCK, D).float() * ratio[..., None, None]
        pages.copy_(held.view(pages.shape).to(torch.float8_e4m3fn))
        scales.copy_(grown)
        ids, off = slot // page, slot % page
        pages.view(torch.uint8)[ids, :, off] = (x / grown[ids, :, off // BLOCK][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    pos = torch.arange(s["N"], device="cuda")
    ids = s["table"][0].long()[pos // page]
    k, v = (_dense(s[n + "_pages"], s[n + "_scales"], ids, pos % page).transpose(0, 1)[None].half().contiguous() for n in "kv")
    return {"k": k, "v": v, "k_scales": s["k_scales"], "v_scales": s["v_scales"]}


def _plain_load(s):
    page, N = s["page"], s["N"]
    pos = torch.arange(N, device="cuda")
    ids = s["table"].long().clamp(min=0)[:, pos // page]                              # [R, N]
    there = (pos < s["ctx"][:, None])[:, None, :, None]
    for name in "kv":
        x = _dense(s[name + "_pages"], s[name + "_scales"], ids, (pos % page).expand_as(ids)).half().transpose(1, 2)      # [R, N, Hkv, D] -> [R, Hkv, N, D]
        s[name + "_out"].copy_(torch.where(there, x, s[name + "_out"]))
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_attn(s):
    R, Hq, Hkv, page, n, C, T = s["R"], s["Hq"], s["Hkv"], s["page"], s["most_new"], s["most_ctx"], s["T"]
    G = Hq // Hkv
    pos = torch.arange(C, device="cuda")
    ids = s["table"].long().clamp(min=0)[:, pos // page]
    there = (pos < s["ctx"][:, None])[:, None, :, None]
    k, v = (torch.where(there, _dense(s[x + "_pages"], s[x + "_scales"], ids, (pos % page).expand_as(ids)).transpose(1, 2), 0) for x in "kv")
    start, new = s["q_start"][:-1].long(), (s["q_start"][1:] - s["q_start"][:-1]).long()
    i = torch.arange(n, device="cuda")
    at = (start[:, None] + i).clamp(max=T - 1)                                        # [R, n]
    q = s["q"][at].float().view(R, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, G * n, D)
    scores = (q @ k.transpose(2, 3).contiguous()).mul_(D ** -0.5).view(R, Hkv, G, n, C)
    p = (s["ctx"].long()[:, None] - new[:, None] + i)[:, None, None, :, None]
    seen = pos <= p
    if s["window"]:
        seen = seen & ((pos > p - s["window"]) | (pos < s["sinks"]))
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1)
    e = torch.exp(scores.sub_(torch.where(top.isfinite(), top, 0.0)[..., None]))
    total = e.sum(-1)
    out = (e.flatten(2, 3) @ v.contiguous()).view(R, Hkv, G, n, D) / torch.where(total > 0, total, 1.0)[..., None]
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(s["q_start"][1:].long().contiguous(), t, right=True)
    real = r * n + t - start[r]                                                       # the tokens' rows of the padded batch
    res = {"out": out.permute(0, 3, 1, 2, 4).reshape(R * n, Hq, D)[real].half()}
    if s["stats"]:
        res["row_max"], res["row_sum"] = (x.permute(0, 3, 1, 2).reshape(R * n, Hq)[real].t().contiguous() for x in (top, total))
    return res


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["op"]
    if not own:
        return {"rope": _plain_rope, "store": _plain_store, "load": _plain_load, "attn": _plain_attn}[op](s)
    import paper_2506_19505_amd as antkv

    if "geom" not in s:
        batch = {"rope": s["R"] or s.get("B"), "store": 1}.get(op, s["R"])
        s["geom"] = antkv.Geometry(batch, s.get("Hq") or s["Hkv"], s["Hkv"], 8)
    if op == "rope":
        if "freqs" not in s:                                     # kept with the weights
            s["freqs"] = antkv.rope_freqs(s["rot"], 10000.0, s["factor"], s["trained"], 1.0, 4.0, device=s["k"].device)
        rows = dict(q_start=s["q_start"], ctx_len=s["ctx"]) if s["R"] else {}
        q, k = antkv.rope(s["geom"], s["q"], s["k"], s["freqs"], style=s["style"], inverse=s["back"], **rows)
        return {"q": q, "k": k} if q is not None else {"k": k}
    pools = s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"]
    if op == "store":
        antkv.qpage_store(s["geom"], s["k"], s["v"], s["slot"], *pools)
        k, v = antkv.qpage_load(s["geom"], *pools, s["table"], s["N"])
        return {"k": k, "v": v, "k_scales": s["k_scales"], "v_scales": s["v_scales"]}
    if op == "load":
        k, v = antkv.qpage_load(s["geom"], *pools, s["table"], s["N"], ctx_len=s["ctx"], k=s["k_out"], v=s["v_out"])
        return {"k": k, "v": v}
    if "workspace" not in s:                                     # kept for the next step, as a server keeps it
        s["workspace"] = antkv.qpage_attn_workspace(s["geom"], s["T"], s["q"].device)
    out, row_max, row_sum = antkv.qpage_attn(s["geom"], s["q"], D ** -0.5, s["q_start"], s["ctx"], s["table"], *pools, window=s["window"],
                                             n_sink=s["sinks"], want_stats=s["stats"], workspace=s["workspace"])
    return {"out": out, "row_max": row_max, "row_sum": row_sum} if s["stats"] else {"out": out}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def _exact_rope(s):
    rot, style, T = s["rot"], s["style"], s["T"]
    f = []
    for i in range(rot // 2):
        x = 10000.0 ** (-2 * i / rot)
        if s["trained"]:
            w = min(1.0, max(0.0, (s["trained"] * x / (2 * math.pi) - 1.0) / 3.0))
            x = w * x + (1 - w) * x / s["factor"]
        else:
            x = x / s["factor"]
        f.append(x)
    if s["R"]:
        starts, ctx = s["q_start"].tolist(), s["ctx"].tolist()
        pos = torch.cat([torch.arange(c - (b - a), c) for a, b, c in zip(starts, starts[1:], ctx)])
    else:
        pos = torch.arange(T)
    turn = torch.outer(pos.double(), torch.tensor(f, dtype=torch.float64)).cuda()
    turn = torch.polar(torch.ones_like(turn), -turn if s["back"] else turn)
    if s["R"]:
        turn = turn[:, None]
    out = {}
    for name in ("q", "k"):
        if s[name] is None:
            continue
        x = s[name].double()
        pair = x[..., :rot].unflatten(-1, (2, rot // 2) if style else (rot // 2, 2)).movedim(-2 if style else -1, -1)
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        x[..., :rot] = z.movedim(-1, -2).flatten(-2) if style else z.flatten(-2)
        out[name] = x
    return out


def _exact_round(y):
    """To the nearest number of three bits behind the first one, exponents from -6 on; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _exact_store(s):
    page, Hkv = s["page"], s["Hkv"]
    slots = s["slot"].long()
    n_pages = s["k_pages"].shape[0]
    out = {}
    for name in "kv":
        held = s[name + "_pages"].float().double().view(n_pages, Hkv, page // BLOCK, BLOCK, D).transpose(1, 2).flatten(0, 1)        # [blocks, Hkv, 16, D]
        scale = s[name + "_scales"].double().transpose(1, 2).flatten(0, 1).clone()                                                 # [blocks, Hkv]
        rows = torch.zeros_like(held)
        new = torch.zeros(held.shape[0], BLOCK, dtype=torch.bool, device="cuda")
        rows.transpose(1, 2)[slots // BLOCK, slots % BLOCK] = s[name].double().clamp(-MOST, MOST)
        new[slots // BLOCK, slots % BLOCK] = True
        amax = rows.abs().amax((2, 3))
        need = torch.full_like(amax, 2.0 ** -32)
        for e in range(-31, 9):
            need = torch.where(amax > 448 * 2.0 ** (e - 1), 2.0 ** e, need)
        grown = torch.where(new[:, :1], need, torch.where(new.any(1)[:, None], torch.maximum(need, scale), scale))
        kept = torch.where(new[:, :1, None, None], held, _exact_round(held * (scale / grown)[..., None, None]))
        got = torch.where(new[:, None, :, None], _exact_round(rows / grown[..., None, None]), kept) * grown[..., None, None]
        got = got.view(n_pages, page // BLOCK, Hkv, BLOCK, D).transpose(1, 2).reshape(n_pages, Hkv, page, D)
        out[name] = torch.cat([got[i] for i in s["table"][0].tolist()], 1)[None]
        out[name + "_scales"] = grown.view(n_pages, page // BLOCK, Hkv).transpose(1, 2).contiguous()
    return out


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


def _exact_head(s, name, pages, g, c):
    """Rows of the first c tokens of a request, KV head g."""
    x = torch.cat([s[name + "_pages"][i, g] for i in pages]).float().double()
    scales = torch.cat([s[name + "_scales"][i, g] for i in pages]).double()
    return (x.view(-1, BLOCK, D) * scales[:, None, None]).view(-1, D)[:c]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "rope":
        return _exact_rope(s)
    if op == "store":
        return _exact_store(s)
    if op == "load":
        out = {x: s[x + "_out"].double() for x in "kv"}
        for r, c in enumerate(s["ctx"].tolist()):
            pages = s["table"][r, :-(-c // s["page"])].tolist()
            for g in range(s["Hkv"]):
                for x in "kv":
                    out[x][r, g, :c] = _exact_head(s, x, pages, g, c)
        return out
    Hq, G, page = s["Hq"], s["Hq"] // s["Hkv"], s["page"]
    starts, ctx = s["q_start"].tolist(), s["ctx"].tolist()
    out = torch.empty((s["T"], Hq, D), dtype=torch.float64, device="cuda")
    top, total = (torch.empty((Hq, s["T"]), dtype=torch.float64, device="cuda") for _ in range(2))
    for r in range(s["R"]):
        a, b, c = starts[r], starts[r + 1], ctx[r]
        pages = s["table"][r, :-(-c // page)].tolist()
        for g in range(s["Hkv"]):
            k, v = _exact_head(s, "k", pages, g, c), _exact_head(s, "v", pages, g, c)
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
    op, Hkv = case["op"], case["Hkv"]
    row, byte_row = 2 * D, D + 4 / BLOCK                         # bytes of a head's row, in fp16 and in 8 bits
    if op == "rope":
        rows = case["B"] * case["T"] * (case["Hq"] + Hkv)
        return {"bytes": rows * 2 * row + 8 * case["R"], "flops": rows * case["rot"] * 3}
    if op == "store":                                            # rows in, blocks out; the pages back
        T, page = case["T"], case["page"]
        rng = random.Random("%(R)d %(T)d" % case)
        held = [rng.randint(1, page) % page for _ in range(case["R"])]
        N = (T + sum(held)) // page * page
        return {"bytes": int(2 * Hkv * (T * (row + byte_row) + N * (row + byte_row)) + 4 * T), "flops": 0}
    if op == "load":
        rows = sum(max(1, case["N"] - 37 * r) for r in range(case["R"]))
        return {"bytes": int(rows * 2 * Hkv * (row + byte_row)), "flops": 0}
    Hq = case["Hq"]
    seen = [_visible(c - n, n, case["window"], case["sinks"]) for c, n in zip(*_lengths(case))]
    pairs, keys = sum(x[0] for x in seen), sum(x[1] for x in seen)
    return {"bytes": int(case["T"] * Hq * (2 * row + (8 if case["stats"] else 0)) + keys * Hkv * 2 * byte_row), "flops": pairs * Hq * 4 * D}
