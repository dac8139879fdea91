"""Performance cases of the operators of a sequence model's block: attention, the root-mean-square norm with
the residual's addition, and rotary positions.

A case is one operator at one size, as a program that trains a trunk or answers with it calls it:

* "attention": `use` "token" (one query a sequence over a cache filled to a length of its own), "prompt" (the
  forward pass alone) or "train" (forward and backward pass); `batch`, `q_len`, `k_len`, `heads`, `kv_heads`,
  `dim`, `type`, and of the scores `causal`, `cap` (0: none), `slopes` (bias by distance), `prefix` (a stretch
  at the start that every query sees), `doc` (mean length of the documents in a row, 0: none).
* "norm": `use` "serve" (x + residual, normalised) or "train" (with the backward pass); `rows`, `width`, `type`,
  `quantize` (the result in 8 bits with a scale a row).
* "rotary": `use` "serve" or "train" (the gradients' rotation too); `batch`, `length`, `heads`, `kv_heads`,
  `dim`, `rot` (the part of the head that turns), `interleaved`, `type`, `first` (the largest first position).

Where `own` is false, `run` computes them in elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


def _attention(name, use, batch, q_len, k_len, heads, kv_heads, dim, type, causal=True, cap=0.0, slopes=False,
               prefix=False, doc=0):
    return {"name": name, "op": "attention", "use": use, "batch": batch, "q_len": q_len, "k_len": k_len, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "type": type, "causal": causal, "cap": cap, "slopes": slopes,
            "prefix": prefix, "doc": doc}


def _norm(name, use, rows, width, type, quantize=False):
    return {"name": name, "op": "norm", "use": use, "rows": rows, "width": width, "type": type, "quantize": quantize}


def _rotary(name, use, batch, length, heads, kv_heads, dim, rot, interleaved, type, first=0):
    return {"name": name, "op": "rotary", "use": use, "batch": batch, "length": length, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "rot": rot, "interleaved": interleaved, "type": type, "first": first}


def listed():
    return [
        # the next token of one short dialogue: only latency counts
        _attention("token_short", "token", 1, 1, 777, 8, 8, 64, "f16", slopes=True),
        # the next tokens of sixteen dialogues over caches filled to lengths of their own, heads in groups of eight
        _attention("tokens_long_cache", "token", 16, 1, 32768, 32, 4, 128, "bf16"),
        # a long prompt read at once
        _attention("prompt_causal", "prompt", 1, 8192, 8192, 16, 4, 128, "bf16"),
        # documents packed into rows of an odd length, capped scores, a head size between the powers of two
        _attention("packed_capped", "prompt", 3, 3001, 3001, 12, 12, 80, "f16", cap=30.0, doc=500),
        # a training step on full rows
        _attention("train_causal", "train", 2, 4096, 4096, 16, 8, 128, "bf16"),
        # a small step in 32 bits with a prefix that is seen in both directions and a bias by distance
        _attention("train_prefix_f32", "train", 2, 513, 513, 8, 2, 64, "f32", slopes=True, prefix=True),
        # the norm before the product of a few tokens, quantised for it
        _norm("norm_tokens_e4m3", "serve", 4, 2048, "bf16", quantize=True),
        # the norm of a batch of prompts
        _norm("norm_prompts", "serve", 16384, 4096, "bf16"),
        # the norm of a training step, forward and backward
        _norm("norm_train", "train", 8192, 2048, "bf16"),
        # the same at sizes that are no multiples of anything, in 32 bits
        _norm("norm_train_odd", "train", 1031, 785, "f32"),
        # the queries' and keys' positions of two long prompts
        _rotary("rotary_prompts", "serve", 2, 8192, 32, 8, 128, 128, False, "bf16", first=4096),
        # interleaved pairs in a part of the head, with the gradients' rotation
        _rotary("rotary_train_part", "train", 3, 1021, 8, 8, 80, 32, True, "f32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "norm", "rotary"))
    if op == "attention":
        use = rng.choice(("token", "prompt", "train"))
        kv_heads = rng.choice((1, 2, 3, 4, 8))
        heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 8))
        dim = rng.choice((32, 64, 64, 72, 80, 96, 128, 128, 128))
        type = rng.choice(("bf16", "bf16", "f16", "f32" if use == "train" else "bf16"))
        batch = _log(rng, 1, 16 if use == "token" else 4)
        length = _log(rng, 33, 32768 if use == "token" else 8192)
        if type == "f32":
            length = min(length, 1500)
        most = 2e8 if use == "train" else 5e8 if use == "prompt" else 1.6e7
        while batch * heads * length * (1 if use == "token" else length) > most or batch * length * kv_heads * dim > 2.5e8:
            length = length * 3 // 4
        q_len = 1 if use == "token" else length
        if use == "prompt" and rng.random() < 0.3:  # the second part of a prompt, over what the cache holds of the first
            q_len = max(2, length // rng.choice((2, 3, 5, 9)))
        causal = rng.random() < 0.85
        return {k: v for k, v in _attention(
            "", use, batch, q_len, length, heads, kv_heads, dim, type, causal, rng.choice((0.0, 0.0, 30.0, 50.0)),
            rng.random() < 0.3, causal and use != "token" and rng.random() < 0.3,
            _log(rng, 40, 2000) if use != "token" and rng.random() < 0.3 else 0).items() if k != "name"}
    if op == "norm":
        use, width = rng.choice(("serve", "serve", "train")), _log(rng, 64, 8192)
        if rng.random() < 0.6:
            width = (width + 7) // 8 * 8
        rows = min(_log(rng, 1, 16384), 67108864 // width)
        return {k: v for k, v in _norm("", use, rows, width, rng.choice(("bf16", "bf16", "f16", "f32")),
                                       use == "serve" and rng.random() < 0.5).items() if k != "name"}
    dim = rng.choice((64, 80, 96, 128, 128))
    return {k: v for k, v in _rotary(
        "", rng.choice(("serve", "train")), _log(rng, 1, 16), _log(rng, 1, 4096), rng.choice((1, 4, 8, 16, 32)),
        rng.choice((1, 2, 4, 8)), dim, rng.choice((dim, dim, dim // 2, 32)), rng.random() < 0.4,
        rng.choice(("bf16", "bf16", "f16", "f32")), _log(rng, 1, 12000)).items() if k != "name"}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["type"]]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * std).to(t)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=g)

    s = {"case": case}
    if case["op"] == "attention":
        b, sq, sk, h, hk, d = (case[k] for k in ("batch", "q_len", "k_len", "heads", "kv_heads", "dim"))
        s["lens"] = s["slopes"] = s["prefix"] = s["docs"] = None
        if sq == sk:  # one projection's output, seen as queries, keys and values
            s["q"], s["k"], s["v"] = normal(b, sq, h + 2 * hk, d).split((h, hk, hk), 2)
        else:
            s["q"], s["k"], s["v"] = normal(b, sq, h, d), normal(b, sk, hk, d), normal(b, sk, hk, d)
        if case["use"] == "token":  # caches filled to between a half and all; what lies behind was never written
            s["lens"] = (sk - (uniform(b) * (sk // 2)).int()).int()
            unfilled = torch.arange(sk, device="cuda") >= s["lens"][:, None]
            s["k"][unfilled] = math.nan
            s["v"][unfilled] = math.nan
        if case["slopes"]:
            s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, h + 1, device="cuda", dtype=torch.float32) / h)
        if case["prefix"]:
            s["prefix"] = (uniform(b) * (sk // 2)).int()
        if case["doc"]:
            s["docs"] = (uniform(b, sk) < 1.0 / case["doc"]).cumsum(1).int()
            s["docs"][:, sk - sk // 16:] = -1  # the row's padding
        if case["use"] == "train":
            s["do"] = normal(b, sq, h, d)
    elif case["op"] == "norm":
        rows, n = case["rows"], case["width"]
        channels = 1.0 + 15.0 * (uniform(n) < 0.01).float()  # a few channels carry large values
        s["x"] = (torch.randn(rows, n, device="cuda", generator=g)).to(t)
        s["residual"] = (2.0 * torch.randn(rows, n, device="cuda", generator=g) * channels).to(t)
        s["weight"] = (1.0 + 0.1 * torch.randn(n, device="cuda", generator=g)).to(t)
        if case["use"] == "train":
            s["dy"], s["dh"] = normal(rows, n), normal(rows, n)
    else:
        b, n, h, hk, d, rot = (case[k] for k in ("batch", "length", "heads", "kv_heads", "dim", "rot"))
        s["q"], s["k"], _ = normal(b, n, h + 2 * hk, d).split((h, hk, hk), 2)
        first = (uniform(b, 1) * (case["first"] + 1)).int()
        s["positions"] = (first + torch.arange(n, device="cuda", dtype=torch.int32)).int().contiguous()
        angle = torch.arange(case["first"] + n + 1, device="cuda", dtype=torch.float64)[:, None] * (
            10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot))
        s["table"] = torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()
        if case["use"] == "train":
            s["dq"], s["dk"] = normal(b, n, h, d), normal(b, n, hk, d)
    return s


# ---- the operators --------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _own(s, case)
    t = TYPES[case["type"]]
    if case["op"] == "attention":
        return _plain_attention(s, case, t)
    if case["op"] == "norm":
        return _plain_norm(s, case, t)
    return _plain_rotary(s, case, t)


def _own(s, case):
    from paper_2206_08720_amd import seq
    if case["op"] == "attention":
        scores = {"causal": case["causal"], "softcap": case["cap"], "slopes": s["slopes"], "k_lens": s["lens"],
                  "prefix": s["prefix"], "docs": s["docs"]}
        if case["use"] != "train":
            return seq.attention(s["q"], s["k"], s["v"], **scores)
        o, lse = seq.attention(s["q"], s["k"], s["v"], return_lse=True, **scores)
        dq, dk, dv = seq.attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, **scores)
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    if case["op"] == "norm":
        if case["quantize"]:
            q, scale, h = seq.rms_norm_e4m3(s["x"], s["weight"], residual=s["residual"], eps=EPS)
            return {"q": q, "scale": scale, "h": h}
        y, h = seq.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        if case["use"] == "serve":
            return {"y": y, "h": h}
        dx, dweight = seq.rms_norm_backward(s["dy"], h, s["weight"], dh=s["dh"], eps=EPS)
        return {"y": y, "h": h, "dx": dx, "dweight": dweight}
    q, k = seq.rotary(s["q"], s["table"], s["positions"], k=s["k"], interleaved=case["interleaved"])
    if case["use"] == "serve":
        return {"q": q, "k": k}
    dq, dk = seq.rotary(s["dq"], s["table"], s["positions"], k=s["dk"], interleaved=case["interleaved"], inverse=True)
    return {"q": q, "k": k, "dq": dq, "dk": dk}


def _visible(s, case):
    """[batch or 1, 1, 1, q_len, k_len]: whether a query sees a key; and the queries' positions [batch or 1, q_len]."""
    sq, sk = case["q_len"], case["k_len"]
    end = torch.full((1,), sk, device="cuda") if s["lens"] is None else s["lens"].long()
    at = end[:, None] - sq + torch.arange(sq, device="cuda")
    j = torch.arange(sk, device="cuda")
    vis = (j < end[:, None])[:, None, :] & (at >= 0)[:, :, None]
    if case["causal"]:
        before = j <= at[:, :, None]
        if s["prefix"] is not None:
            before = before | (j < s["prefix"].long()[:, None])[:, None, :]
        vis = vis & before
    if s["docs"] is not None:
        docs = s["docs"]
        mine = docs.gather(1, at.clamp(0, sk - 1).expand(case["batch"], sq))
        vis = vis & (mine[:, :, None] == docs[:, None, :]) & (docs >= 0)[:, None, :]
    return vis[:, None, None], at


def _plain_attention(s, case, t):
    b, sq, sk, h, hk, d = (case[k] for k in ("batch", "q_len", "k_len", "heads", "kv_heads", "dim"))
    grp, scale, cap = h // hk, 1.0 / math.sqrt(case["dim"]), case["cap"]
    vis, at = _visible(s, case)

    def rows(x):  # [batch, q_len, heads, dim] -> [batch, kv_heads, group * q_len, dim]
        return x.float().view(b, sq, hk, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * sq, d)

    def unrows(x):
        return x.view(b, hk, grp, sq, d).permute(0, 3, 1, 2, 4).reshape(b, sq, h, d).to(t)

    q, k, v = rows(s["q"]), s["k"].float().transpose(1, 2), s["v"].float().transpose(1, 2)
    if s["lens"] is not None:
        filled = (torch.arange(sk, device="cuda") < s["lens"][:, None])[:, None, :, None]
        k, v = torch.where(filled, k, 0.0), torch.where(filled, v, 0.0)
    k, v = k.contiguous(), v.contiguous()
    x = torch.matmul(q, k.transpose(2, 3)).view(b, hk, grp, sq, sk).mul_(scale)
    capped = (x / cap).tanh_() if cap else None
    if cap:
        x = capped * cap
    if s["slopes"] is not None:
        far = (at[:, :, None] - torch.arange(sk, device="cuda")).abs().float()
        x = x - s["slopes"].view(hk, grp, 1, 1) * far[:, None, None]
    x = x.masked_fill(~vis, -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = (x - top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p / total.clamp_min(torch.finfo(torch.float32).tiny)
    del x
    o32 = torch.matmul(p.view(b, hk, grp * sq, sk), v)
    o = unrows(o32)
    if case["use"] != "train":
        return o
    lse = (total.log() + top).reshape(b, h, sq)
    do = rows(s["do"])
    pm = p.view(b, hk, grp * sq, sk)
    dv = torch.matmul(pm.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_((do * o32).sum(-1, keepdim=True)).mul_(pm)
    if cap:
        ds = ds * (1.0 - capped * capped).view(ds.shape)
    ds = ds.mul_(scale)
    return {"o": o, "lse": lse, "dq": unrows(torch.matmul(ds, k)),
            "dk": torch.matmul(ds.transpose(2, 3), q).transpose(1, 2).to(t).contiguous(),
            "dv": dv.transpose(1, 2).to(t).contiguous()}


def _plain_norm(s, case, t):
    h, w = s["x"].float() + s["residual"].float(), s["weight"].float()
    r = ((h * h).mean(-1, keepdim=True) + EPS).rsqrt()
    y = h * r * w
    if case["quantize"]:
        most = y.abs().amax(-1, keepdim=True)
        scale = torch.where(most > 0, most / 448.0, 1.0)
        return {"q": (y / scale).to(torch.float8_e4m3fn), "scale": scale[:, 0], "h": h.to(t)}
    if case["use"] == "serve":
        return {"y": y.to(t), "h": h.to(t)}
    dy = s["dy"].float()
    g = dy * w
    dx = r * (g - h * (r * r) * (g * h).mean(-1, keepdim=True)) + s["dh"].float()
    return {"y": y.to(t), "h": h.to(t), "dx": dx.to(t), "dweight": (dy * h * r).sum(0).to(t)}


def _plain_rotary(s, case, t):
    turn = s["table"][s["positions"].long()]  # [batch, length, rot / 2, 2]
    c, sn = turn[:, :, None, :, 0], turn[:, :, None, :, 1]
    rot = case["rot"]

    def rotate(x, sn):
        a = x[..., :rot].float()
        u, v = (a[..., 0::2], a[..., 1::2]) if case["interleaved"] else (a[..., :rot // 2], a[..., rot // 2:])
        u, v = u * c - v * sn, v * c + u * sn
        a = torch.stack((u, v), -1).flatten(-2) if case["interleaved"] else torch.cat((u, v), -1)
        return torch.cat((a.to(t), x[..., rot:]), -1)

    got = {"q": rotate(s["q"], sn), "k": rotate(s["k"], sn)}
    if case["use"] == "train":
        got.update(dq=rotate(s["dq"], -sn), dk=rotate(s["dk"], -sn))
    return got


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x, res, w = (s[k].double() for k in ("x", "residual", "weight"))
        h, w = (x + res).requires_grad_(), w.requires_grad_()
        y = h / torch.sqrt(torch.sum(h ** 2, 1, keepdim=True) / case["width"] + EPS) * w
        if case["quantize"]:
            scale = y.abs().max(1).values / 448
            return {"q": (y / scale[:, None]).detach(), "scale": scale.detach(), "h": h.detach()}
        if case["use"] == "serve":
            return {"y": y.detach(), "h": h.detach()}
        dh, dw = torch.autograd.grad([y, h * 1], [h, w], [s["dy"].double(), s["dh"].double()])
        return {"y": y.detach(), "h": h.detach(), "dx": dh, "dweight": dw}
    if case["op"] == "rotary":
        table = s["table"].double()[s["positions"].reshape(-1).long()]
        z = torch.complex(table[..., 0], table[..., 1]).view(case["batch"], case["length"], 1, -1)

        def turned(x, z):
            out, rot = x.double(), case["rot"]
            even = torch.arange(0, rot, 2, device="cuda") if case["interleaved"] else torch.arange(rot // 2, device="cuda")
            odd = even + 1 if case["interleaved"] else even + rot // 2
            w = torch.complex(out[..., even], out[..., odd]) * z
            out = out.clone()
            out[..., even], out[..., odd] = w.real, w.imag
            return out

        got = {"q": turned(s["q"], z), "k": turned(s["k"], z)}
        if case["use"] == "train":
            got.update(dq=turned(s["dq"], z.conj()), dk=turned(s["dk"], z.conj()))
        return got
    return _exact_attention(s, case)


def _exact_attention(s, case):
    sq, sk, h, hk = (case[k] for k in ("q_len", "k_len", "heads", "kv_heads"))
    train = case["use"] == "train"
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["batch"], h, sq, dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("q", "k", "v"))
    for b in range(case["batch"]):
        end = sk if s["lens"] is None else int(s["lens"][b])
        i, j = torch.arange(end - sq, end, device="cuda")[:, None], torch.arange(end, device="cuda")[None, :]
        seen = (i >= 0).expand(sq, end)
        if case["causal"]:
            seen = seen & ((i >= j) | (j < (0 if s["prefix"] is None else int(s["prefix"][b]))))
        if s["docs"] is not None:
            ids = s["docs"][b, :end]
            seen = seen & (ids[i.clamp_min(0)] == ids[j]) & (ids[j] >= 0)
        some = seen.any(1, keepdim=True)
        for a in range(h):
            c = a // (h // hk)
            q, k, v = s["q"][b, :, a].double(), s["k"][b, :end, c].double(), s["v"][b, :end, c].double()
            if train:
                q, k, v = q.requires_grad_(), k.requires_grad_(), v.requires_grad_()
            z = q @ k.T / math.sqrt(case["dim"])
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if s["slopes"] is not None:
                z = z - s["slopes"][a].double() * (i - j).abs()
            z = torch.where(seen, z, torch.where(some, -math.inf, 0.0))
            w = torch.softmax(z, 1) * some
            y = w @ v
            o[b, :, a] = y.detach()
            if train:
                lse[b, a] = torch.where(some[:, 0], torch.logsumexp(z, 1), -math.inf).detach()
                gq, gk, gv = torch.autograd.grad(y, [q, k, v], s["do"][b, :, a].double())
                dq[b, :, a] = gq
                dk[b, :end, c] += gk
                dv[b, :end, c] += gv
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if train else o


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def _pairs(case):
    """Visible (query, key) pairs of one row of the batch, the mean over what prepare() draws."""
    sq, sk, m = case["q_len"], case["k_len"], case["doc"]
    if case["use"] == "token":
        return 0.75 * sk
    causal = sq * (sk - sq) + sq * (sq + 1) / 2.0
    if m:  # a pair at distance n lies in one document with probability (1 - 1/m)^n
        stay, live = 1.0 - 1.0 / m, sk - sk // 16
        causal = sum(m * (1.0 - stay ** (i + 1)) for i in range(max(0, sk - sq), live))
        return causal if case["causal"] else 2.0 * causal - max(0, live - max(0, sk - sq))
    if not case["causal"]:
        return float(sq) * sk
    return causal + (sk * sk / 24.0 if case["prefix"] and sq == sk else 0.0)


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["type"]]
    train = case["use"] == "train"
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        if case["quantize"]:
            return {"bytes": n * (3 * size + 1) + 4 * case["rows"], "flops": 6 * n}
        return {"bytes": n * size * (8 if train else 4), "flops": (16 if train else 6) * n}
    if case["op"] == "rotary":
        n = case["batch"] * case["length"]
        heads = n * (case["heads"] + case["kv_heads"])
        table = 4 * case["rot"] * min(n, case["first"] + case["length"])
        return {"bytes": (2 * heads * case["dim"] * size) * (2 if train else 1) + table, "flops": 3 * heads * case["rot"] * (2 if train else 1)}
    b, d = case["batch"], case["dim"]
    q = b * case["q_len"] * case["heads"] * d * size
    kv = b * case["k_len"] * case["kv_heads"] * d * size * 2 * (0.75 if case["use"] == "token" else 1)
    flops = b * case["heads"] * _pairs(case) * d * (14 if train else 4)
    return {"bytes": (4 * q + 2 * kv) if train else (2 * q + kv), "flops": flops}
