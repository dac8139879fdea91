"""Performance cases of the operators that a sequence model answers with: appending keys and values to a cache that
lies in pages, attention over that cache, and the log probabilities of the tokens that come out.

A case is one operator at one size, as a program that answers with a model, or trains on its answers, calls it:

* "append": the new tokens' keys turn to their positions and go into the cache with the values, and the queries turn; `batch`,
  `length` (new tokens a sequence; over 1: between half and all of them are there), `held` (the most tokens that
  a sequence held before), `heads`, `kv_heads`, `dim`, `rot` (the part of the head that turns, 0: none),
  `interleaved`, `type`, `e4m3` (the cache in 8 bits, under a power of two for each page and head), `page`.
* "attention": `batch`, `q_len` (1: the next token; a few: drafts; many: a part of a prompt, of which between half and all is there),
  `k_len` (the longest sequence in the cache), `heads`, `kv_heads`, `dim`, `type`, `e4m3`, `page`, and of the scores `cap` (0:
  none) and `slopes` (bias by distance).
* "logprobs": `use` "serve" or "train" (with the gradient), `rows`, `vocab`, `type`, `top` (alternatives asked
  for), `scale` (one over the temperature).

Where `own` is false, `run` computes them in elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn


def _append(name, batch, length, held, heads, kv_heads, dim, rot, interleaved, type, e4m3, page):
    return {"name": name, "op": "append", "batch": batch, "length": length, "held": held, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "rot": rot, "interleaved": interleaved, "type": type, "e4m3": e4m3, "page": page}


def _attention(name, batch, q_len, k_len, heads, kv_heads, dim, type, e4m3, page, cap=0.0, slopes=False):
    return {"name": name, "op": "attention", "batch": batch, "q_len": q_len, "k_len": k_len, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "type": type, "e4m3": e4m3, "page": page, "cap": cap, "slopes": slopes}


def _logprobs(name, use, rows, vocab, type, top=0, scale=1.0):
    return {"name": name, "op": "logprobs", "use": use, "rows": rows, "vocab": vocab, "type": type, "top": top, "scale": scale}


def listed():
    return [
        # the next tokens of 64 dialogues, into a cache in 8 bits: only latency counts
        _append("append_tokens_e4m3", 64, 1, 8192, 32, 8, 128, 128, False, "bf16", True, 64),
        # four prompts read at once, in small pages
        _append("append_prompts", 4, 4096, 0, 32, 8, 128, 128, False, "bf16", False, 16),
        # second parts of prompts that begin within a page; part of the head turns, by interleaved pairs
        _append("append_parts_e4m3", 3, 1021, 777, 8, 8, 80, 32, True, "f16", True, 32),
        # the next token of one short dialogue
        _attention("token_short", 1, 1, 777, 8, 8, 64, "f16", False, 16, slopes=True),
        # the next tokens of 96 dialogues, in small pages
        _attention("tokens_many", 96, 1, 4096, 32, 8, 128, "bf16", False, 16),
        # the next tokens of 32 long dialogues, in 8 bits
        _attention("tokens_long_e4m3", 32, 1, 32768, 32, 4, 128, "bf16", True, 64),
        # five drafted tokens a dialogue, checked at once
        _attention("drafts_e4m3", 16, 5, 8192, 16, 2, 128, "bf16", True, 32),
        # parts of two long prompts over what the cache holds of them
        _attention("part_e4m3", 2, 2048, 16384, 32, 8, 128, "bf16", True, 64),
        # an odd part of three shorter ones, with capped scores, a bias by distance and a head size between the powers of two
        _attention("part_capped", 3, 501, 3001, 12, 12, 80, "f16", False, 32, cap=30.0, slopes=True),
        # the tokens that eight dialogues answered with, and twenty alternatives to each
        _logprobs("answers_top", "serve", 8, 131072, "bf16", top=20, scale=1.0 / 0.7),
        # a training step on the tokens of a batch, with the entropy's gradient
        _logprobs("train_tokens", "train", 4096, 65536, "bf16"),
        # the same in 32 bits at sizes that are no multiples of anything
        _logprobs("train_tokens_odd", "train", 1031, 50001, "f32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "attention", "attention", "logprobs"))
    if op == "logprobs":
        use, vocab = rng.choice(("serve", "train")), _log(rng, 500, 131072)
        rows = min(_log(rng, 1, 4096), 134217728 // vocab)
        return {k: v for k, v in _logprobs("", use, rows, vocab, rng.choice(("bf16", "bf16", "f16", "f32")),
                                           rng.choice((0, 1, 5, 20)), rng.choice((1.0, 1.25, 0.5))).items() if k != "name"}
    kv_heads = rng.choice((1, 2, 3, 4, 8))
    heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 8))
    dim = rng.choice((32, 64, 64, 72, 80, 96, 128, 128, 128))
    type, page = rng.choice(("bf16", "bf16", "bf16", "f16", "f16", "f32")), rng.choice((8, 16, 32, 64, 128))
    e4m3 = rng.random() < 0.5
    if op == "append":
        length = rng.choice((1, 1, _log(rng, 2, 4096)))
        batch = _log(rng, 1, 128 if length == 1 else 4)
        return {k: v for k, v in _append("", batch, length, _log(rng, 1, 8192), heads, kv_heads, dim, rng.choice((dim, dim, dim // 2, 32, 0)),
                                         rng.random() < 0.3, type, e4m3, page).items() if k != "name"}
    q_len = rng.choice((1, 1, rng.randint(2, 8), _log(rng, 9, 2048)))
    batch, k_len = _log(rng, 1, 64 if q_len == 1 else 16 if q_len < 9 else 3), max(q_len, _log(rng, 33, 32768))
    while batch * heads * float(k_len) * q_len * (dim / 128) > (5e8 if type != "f32" else 1e8) or batch * k_len * kv_heads * dim > 2.5e8:
        k_len = max(1, k_len * 3 // 4)
        q_len = min(q_len, k_len)
    return {k: v for k, v in _attention("", batch, q_len, k_len, heads, kv_heads, dim, type, e4m3, page,
                                        rng.choice((0.0, 0.0, 30.0, 50.0)), rng.random() < 0.3).items() if k != "name"}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _power(most):
    """The least power of two (at least 2^-126) that `most` is at most 448 times of."""
    m, e = torch.frexp(most)
    return torch.where(most > 0, torch.ldexp(torch.ones_like(most), torch.where(m <= 0.875, e - 9, e - 8).clamp_min(-126)), 2.0 ** -126)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["type"]]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * std).to(t)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=g)

    s = {"case": case}
    if case["op"] == "logprobs":
        rows, n = case["rows"], case["vocab"]
        s["logits"] = normal(rows, n, std=2.5)
        s["tokens"] = (uniform(rows) * n).int().clamp_max(n - 1)
        likely = uniform(rows) < 0.8  # most of the tokens are ones that the model expects
        at = torch.arange(rows, device="cuda")[likely]
        s["logits"][at, s["tokens"][likely].long()] = normal(at.numel(), std=2.0) + 10.0
        if case["use"] == "train":
            s["tokens"][uniform(rows) < 0.05] = -1  # prompts and padding
            s["dlogp"], s["dentropy"] = -torch.randn(rows, device="cuda", generator=g) / rows, torch.full((rows,), -0.01 / rows, device="cuda")
        return s
    b, h, hk, d, page = (case[k] for k in ("batch", "heads", "kv_heads", "dim", "page"))
    append = case["op"] == "append"
    n, most = (case["length"], case["held"] + case["length"]) if append else (case["q_len"], case["k_len"])
    # sequences of lengths of their own; their pages lie anywhere, some are free, and what is behind the last token was
    # never written (it holds NaN; zeros where a case returns the whole cache)
    per = -(-most // page)
    count = b * per + b * per // 50 + 1
    s["new"] = (n - (uniform(b) * (n // 2)).int()).int() if n > 1 else torch.ones(b, dtype=torch.int32, device="cuda")
    if append:
        s["lens"] = (case["held"] - (uniform(b) * (case["held"] // 2 + 1)).int()).int()
        total = s["lens"] + s["new"]
    else:
        total = torch.maximum(most - (uniform(b) * (most // 2)).int(), s["new"]).int()
        s["lens"] = total
    there = torch.arange(per, device="cuda") * page < total[:, None]
    s["pages"] = torch.where(there, torch.randperm(count, device="cuda", generator=g)[:b * per].view(b, per), -1).int().contiguous()
    # [pages, page, kv_heads, dim], each head's part of a page in one piece
    held_pages = torch.arange(per, device="cuda") * page < s["lens"][:, None]
    s["k_scale"] = s["v_scale"] = None
    for name in ("k", "v"):
        x = torch.randn(count, hk, page, d, device="cuda", generator=g)
        if case["e4m3"]:
            scale = _power(x.abs().amax((2, 3)))
            cells = (x / scale[:, :, None, None]).to(E4M3)
            s[name + "_scale"] = scale
            cells, empty = cells.view(torch.uint8), 0x7f
        else:
            cells, empty = x.to(t), math.nan
        inside = torch.zeros(count, page, dtype=torch.bool, device="cuda")
        slots = torch.arange(per * page, device="cuda").view(per, page) < s["lens"][:, None, None]
        inside[s["pages"][held_pages].long()] = slots[held_pages]
        cells.masked_fill_(~inside[:, None, :, None], 0 if append else empty)
        s[name + "_cache"] = (cells.view(E4M3) if case["e4m3"] else cells).transpose(1, 2)
        del x, cells
    if append:
        # one projection's output, seen as queries, keys and values
        s["q"], s["k"], s["v"] = normal(b, n, h + 2 * hk, d).split((h, hk, hk), 2)
        s["table"] = None
        if case["rot"]:
            angle = torch.arange(most + 1, device="cuda", dtype=torch.float64)[:, None] * (
                10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"]))
            s["table"] = torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()
        return s
    s["q"] = normal(b, n, h, d)
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, h + 1, device="cuda", dtype=torch.float32) / h) if case["slopes"] else None
    return s


# ---- the operators --------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _own(s, case)
    return {"append": _plain_append, "attention": _plain_attention, "logprobs": _plain_logprobs}[case["op"]](s, case, TYPES[case["type"]])


def _updated(s, q):
    return {"q": q, "k": s["k_cache"], "v": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]} if s["case"]["e4m3"] else {
        "q": q, "k": s["k_cache"], "v": s["v_cache"]}


def _own(s, case):
    from paper_2206_08720_amd import seq
    if case["op"] == "logprobs":
        got = seq.token_logprobs(s["logits"], s["tokens"], top=case["top"], scale=case["scale"])
        out = {"logp": got.logp, "entropy": got.entropy}
        if case["top"]:
            out.update(top_logp=got.top_logp, top_tokens=got.top_tokens)
        if case["use"] == "train":
            out["dlogits"] = seq.token_logprobs_backward(s["dlogp"], s["dentropy"], s["logits"], s["tokens"], got.lse, got.entropy,
                                                         scale=case["scale"])
        return out
    cache = seq.PagedCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    if case["op"] == "append":
        q = seq.cache_append(cache, s["pages"], s["lens"], s["k"], s["v"], q=s["q"], table=s["table"], new_lens=s["new"],
                             interleaved=case["interleaved"])
        return _updated(s, q)
    return seq.attention_cached(s["q"], cache, s["pages"], s["lens"], q_lens=s["new"], softcap=case["cap"], slopes=s["slopes"])


def _turned(x, turn, rot, interleaved):
    """The heads of x [batch, length, heads, dim] in 32 bits, turned by turn [batch, length, rot / 2, 2]."""
    x = x.float()
    if not rot:
        return x
    c, sn = turn[:, :, None, :, 0], turn[:, :, None, :, 1]
    a = x[..., :rot]
    u, v = (a[..., 0::2], a[..., 1::2]) if interleaved else (a[..., :rot // 2], a[..., rot // 2:])
    u, v = u * c - v * sn, v * c + u * sn
    a = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((a, x[..., rot:]), -1)


def _plain_append(s, case, t):
    n, page = case["length"], case["page"]
    at = s["lens"][:, None] + torch.arange(n, device="cuda")  # [batch, length]
    there = torch.arange(n, device="cuda") < s["new"][:, None]
    turn = None if s["table"] is None else s["table"][torch.where(there, at, 0).long()]
    q = torch.where(there[:, :, None, None], _turned(s["q"], turn, case["rot"], case["interleaved"]), 0.0).to(t)
    row, i = there.nonzero(as_tuple=True)
    pos = at[row, i].long()
    cell = s["pages"][row, pos // page].long(), pos % page
    for name in ("k", "v"):
        new = _turned(s[name], turn, case["rot"] if name == "k" else 0, case["interleaved"])[row, i]  # [tokens, kv_heads, dim]
        cache = s[name + "_cache"]
        if not case["e4m3"]:
            cache[cell] = new.to(t)
            continue
        scale = s[name + "_scale"]
        first = (s["lens"] // page).long()  # the page that a sequence's first new token comes into: it may hold older ones
        begun, held = (s["lens"] % page > 0) & (s["new"] > 0), s["lens"] % page
        begun_page = s["pages"].gather(1, first.clamp_max(s["pages"].shape[1] - 1)[:, None])[:, 0].long()[begun]
        old_scale = scale[begun_page]
        most = torch.zeros_like(scale).index_reduce_(0, cell[0], new.abs().amax(-1), "amax")
        touched = torch.zeros(scale.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, cell[0], True)
        now = _power(most)
        now[begun_page] = torch.maximum(now[begun_page], old_scale)
        scale.copy_(torch.where(touched[:, None], now, scale))
        older = torch.arange(page, device="cuda") < held[begun][:, None]
        cells = cache[begun_page].float() * (old_scale / scale[begun_page])[:, None, :, None]
        cache.view(torch.uint8)[begun_page] = torch.where(older[:, :, None, None], cells.to(E4M3).view(torch.uint8),
                                                          cache.view(torch.uint8)[begun_page])
        cache.view(torch.uint8)[cell] = (new / scale[cell[0]][:, :, None]).to(E4M3).view(torch.uint8)
    return _updated(s, q)


def _contents(s, case, name, type):
    """Every sequence's keys or values [batch, places, kv_heads, dim], zeros where none are."""
    pages = s["pages"].long().clamp_min(0)
    x = s[name + "_cache"][pages].to(type)  # [batch, pages, page, kv_heads, dim]
    if case["e4m3"]:
        x = x * s[name + "_scale"][pages].to(type)[:, :, None, :, None]
    x = x.flatten(1, 2)
    return x.masked_fill_((torch.arange(x.shape[1], device="cuda") >= s["lens"][:, None])[:, :, None, None], 0.0)


def _plain_attention(s, case, t):
    b, sq, h, hk, d = (case[k] for k in ("batch", "q_len", "heads", "kv_heads", "dim"))
    grp, cap = h // hk, case["cap"]
    k, v = (_contents(s, case, name, torch.float32).transpose(1, 2).contiguous() for name in ("k", "v"))
    sk = k.shape[2]
    q = s["q"].float().view(b, sq, hk, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * sq, d)
    i, j = torch.arange(sq, device="cuda"), torch.arange(sk, device="cuda")
    at = torch.where(i < s["new"][:, None], (s["lens"] - s["new"])[:, None] + i, -1)  # [batch, q_len]
    x = torch.matmul(q, k.transpose(2, 3)).view(b, hk, grp, sq, sk).mul_(1.0 / math.sqrt(d))
    if cap:
        x = x.div_(cap).tanh_().mul_(cap)
    if s["slopes"] is not None:
        x = x - s["slopes"].view(hk, grp, 1, 1) * (at[:, :, None] - j).abs().float()[:, None, None]
    x = x.masked_fill_((j > at[:, :, None])[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = x.sub_(top).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).tiny))
    o = torch.matmul(p.view(b, hk, grp * sq, sk), v)
    return o.view(b, hk, grp, sq, d).permute(0, 3, 1, 2, 4).reshape(b, sq, h, d).to(t)


def _plain_logprobs(s, case, t):
    x, n = s["logits"].float() * case["scale"], case["vocab"]
    top = x.amax(1, keepdim=True)
    e = (x - top).exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    mean = (e * torch.where(e > 0, x - top, 0.0)).sum(1, keepdim=True) / total
    entropy, lse = (log_total - mean)[:, 0], top + log_total
    there = s["tokens"] >= 0
    token = s["tokens"].clamp_min(0).long()[:, None]
    out = {"logp": torch.where(there, (x.gather(1, token) - top - log_total)[:, 0], 0.0), "entropy": entropy}
    if case["top"]:
        # the largest first, and of equal ones the lowest token: one whole number holds both
        bits = (s["logits"].float() + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * 4294967296 + (n - 1 - torch.arange(n, device="cuda"))
        which = n - 1 - key.topk(min(case["top"], n), 1).values % 4294967296
        out.update(top_logp=x.gather(1, which) - top - log_total, top_tokens=which.int())
    if case["use"] == "train":
        logp = x - lse
        p = logp.exp()
        dlogp = torch.where(there, s["dlogp"], 0.0)[:, None]
        d = p * (-dlogp - s["dentropy"][:, None] * torch.where(p > 0, logp + entropy[:, None], 0.0))
        out["dlogits"] = d.scatter_add_(1, token, dlogp).mul_(case["scale"]).to(t)
    return out


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "logprobs": _exact_logprobs}[case["op"]](s, case)


def _exact_append(s, case):
    rot, page = case["rot"], case["page"]
    even = torch.arange(0, rot, 2, device="cuda") if case["interleaved"] else torch.arange(rot // 2, device="cuda")
    odd = even + 1 if case["interleaved"] else even + rot // 2

    def turned(x, first):
        x = x.double().clone()
        if rot:
            table = s["table"][first:first + x.shape[0]].double()
            z = torch.complex(x[..., even], x[..., odd]) * torch.complex(table[..., 0], table[..., 1])[:, None]
            x[..., even], x[..., odd] = z.real, z.imag
        return x

    got = {"q": torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")}
    for name in ("k", "v"):
        cells, scale = s[name + "_cache"].double(), s[name + "_scale"].double() if case["e4m3"] else None
        for b in range(case["batch"]):
            first, n = int(s["lens"][b]), int(s["new"][b])
            if name == "k":
                got["q"][b, :n] = turned(s["q"][b, :n], first)
            new = turned(s["k"][b, :n], first) if name == "k" else s["v"][b, :n].double()
            for at in range(first // page, (first + n - 1) // page + 1):
                lo, hi = max(first, at * page), min(first + n, (at + 1) * page)
                where, part = int(s["pages"][b, at]), new[lo - first:hi - first]
                if case["e4m3"]:
                    now = 2.0 ** (part.abs().amax((0, 2)) / 448).log2().ceil()
                    if lo > at * page:
                        now = torch.maximum(now, scale[where])
                        cells[where, :lo - at * page] *= (scale[where] / now)[:, None]
                    scale[where] = now
                    part = part / now[:, None]
                cells[where, lo - at * page:hi - at * page] = part
        got[name] = cells
        if case["e4m3"]:
            got[name + "_scale"] = scale
    return got


def _exact_attention(s, case):
    h, hk = case["heads"], case["kv_heads"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        end, n = int(s["lens"][b]), int(s["new"][b])
        where = torch.arange(end, device="cuda")
        page = s["pages"][b, where // case["page"]].long()
        i = torch.arange(end - n, end, device="cuda")[:, None]
        for c in range(hk):
            k, v = (s[name + "_cache"][page, where % case["page"], c].double() for name in ("k", "v"))
            if case["e4m3"]:
                k, v = k * s["k_scale"][page, c].double()[:, None], v * s["v_scale"][page, c].double()[:, None]
            for a in range(c * (h // hk), (c + 1) * (h // hk)):
                z = s["q"][b, :n, a].double() @ k.T / math.sqrt(case["dim"])
                if case["cap"]:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][a].double() * (i - where).abs()
                o[b, :n, a] = torch.softmax(torch.where(where <= i, z, -math.inf), 1) @ v
    return o


def _exact_logprobs(s, case):
    rows, n, top, train = case["rows"], case["vocab"], case["top"], case["use"] == "train"
    parts = []
    step = max(1, 2 ** 26 // n)
    for r in range(0, rows, step):
        logits, tokens = s["logits"][r:r + step], s["tokens"][r:r + step].long()
        x = logits.double().requires_grad_()
        logp = torch.log_softmax(x * case["scale"], 1)
        entropy = -(logp.exp() * logp).sum(1)
        mine = torch.where(tokens >= 0, logp[torch.arange(len(tokens), device="cuda"), tokens.clamp_min(0)], 0.0)
        got = {"logp": mine.detach(), "entropy": entropy.detach()}
        if top:
            which = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :top]
            got.update(top_logp=logp.detach().gather(1, which), top_tokens=which.int())
        if train:
            got["dlogits"], = torch.autograd.grad([mine, entropy], x, [s["dlogp"][r:r + step].double(), s["dentropy"][r:r + step].double()])
        parts.append(got)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["type"]]
    if case["op"] == "logprobs":
        n, train = case["rows"] * case["vocab"], case["use"] == "train"
        return {"bytes": n * size * (3 if train else 1) + case["rows"] * (12 + 8 * case["top"] + (16 if train else 0)),
                "flops": (14 if train else 6) * n}
    b, d, hk, h = (case[k] for k in ("batch", "dim", "kv_heads", "heads"))
    new = case["length"] if case["op"] == "append" else case["q_len"]
    new = float(b) * (new if new == 1 else 0.75 * new)  # the mean of what prepare() draws
    cell = 1 if case["e4m3"] else size
    if case["op"] == "append":
        table = 4 * case["rot"] * min(new, case["held"] + case["length"])
        return {"bytes": int(new * d * (2 * h * size + 2 * hk * (size + cell)) + table),
                "flops": int(3 * new * (h + hk) * case["rot"] + (4 * new * hk * d if case["e4m3"] else 0))}
    keys, n = 0.75 * case["k_len"], new / b
    pairs = n * max(0.0, keys - n) + n * (n + 1) / 2.0
    return {"bytes": int(2 * new * h * d * size + 2 * b * keys * hk * d * cell), "flops": int(4 * b * h * d * pairs)}
