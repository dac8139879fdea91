"""The operators of a sequence model's block (paper_2206_08720_amd.seq) against their definitions in 64 bits.

Tolerances follow from the arithmetic.  u is the type's unit roundoff (fp32 2^-24, bf16 2^-8, fp16 2^-11) and e = 2^-24 that of
the fp32 sums.  An output y is rounded once: u |y| (fp16: 2^-25 more, half its smallest step).  What goes before, first order:
* norm: n-term fp32 sums of squares and products, relative error at most (n + 8) e of the sums of magnitudes;
* attention: the scores' sums of D products, |ds| <= (D + 8) e sum|q k| scale (plus 8 e cap with a cap), change a
  probability by the relative kappa = 2 max|ds| + (k_len + 8) e; p and ds are rounded to the type (u each,
  fp16 also by its smallest step 2^-25) for their products with v, dout, k and q.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}


def _types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _rand(shape, seed, type="f32", std=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(_types()[type])


def _close(name, got, ref, tol):
    import torch
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got)), f"{name}: finite in other places"
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)]), name
    over = ((got - ref).abs() - tol)[fine]
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 0.0, f"{name}: {worst:.3e} over the tolerance"


# ---- attention ------------------------------------------------------------------------------------------------------

def _oracle(q, k, v, type, do=None, causal=False, softcap=0.0, scale=None, slopes=None, k_lens=None, prefix=None, docs=None, inner=None):
    """{name: (value, tolerance)} in 64 bits on the CPU; a hidden pair enters no sum.  inner: the smallest step of p and
    ds in their products (the type's own, where the kernels do not scale them)."""
    import torch
    u, tiny = U[type], TINY[type]
    inner = tiny if inner is None else inner
    B, Sq, H, D = q.shape
    Sk, Hk = k.shape[1], k.shape[2]
    scale = 1 / math.sqrt(D) if scale is None else scale
    q, k, v = q.double(), k.double(), v.double()
    z = torch.zeros
    out = {"o": [z(B, Sq, H, D).double(), z(B, Sq, H, D).double()], "lse": [z(B, H, Sq).double(), z(B, H, Sq).double()]}
    if do is not None:
        do = do.double()
        out["dq"] = [z(B, Sq, H, D).double(), z(B, Sq, H, D).double()]
        for n in ("dk", "dv"):
            out[n] = [z(B, Sk, Hk, D).double(), z(B, Sk, Hk, D).double()]
    for b in range(B):
        n = Sk if k_lens is None else min(max(int(k_lens[b]), 0), Sk)
        pos = n - Sq + torch.arange(Sq)[:, None]
        j = torch.arange(Sk)[None]
        vis = (j < n) & (pos >= 0)
        if causal:
            vis = vis & ((j <= pos) | (j < (0 if prefix is None else int(prefix[b]))))
        if docs is not None:
            mine = docs[b][pos.clamp(0, max(Sk - 1, 0))] if Sk else z(Sq, 1)
            vis = vis & (mine == docs[b][None]) & (docs[b][None] >= 0)
        some = vis.any(1)
        for h in range(H):
            c = h // (H // Hk)
            # what nobody sees leaves the sums before anything is multiplied
            qq = torch.where(some[:, None], q[b, :, h], 0.0)
            seen = vis.any(0)
            kk, vv = torch.where(seen[:, None], k[b, :, c], 0.0), torch.where(seen[:, None], v[b, :, c], 0.0)
            raw = (qq @ kk.T) * scale
            mag = (qq.abs() @ kk.abs().T) * scale
            t = torch.tanh(raw / softcap) if softcap else None
            s = softcap * t if softcap else raw
            fac = 1 - t * t if softcap else torch.ones_like(raw)
            if slopes is not None:
                s = s - slopes[h].double() * (pos - j).abs()
                mag = mag + slopes[h].double() * (pos - j).abs()
            s = torch.where(vis, s, -math.inf)
            top = torch.where(some, s.max(1).values if Sk else z(Sq).double(), 0.0)
            ex = torch.where(vis, torch.exp(s - top[:, None]), 0.0)
            l = ex.sum(1)
            P = ex / torch.where(some, l, 1.0)[:, None]
            dscore = torch.where(vis, (D + 8) * E * mag + 8 * E * softcap, 0.0).max() if Sk else 0.0
            kappa = 2 * float(dscore) + (Sk + 8) * E
            o = P @ vv
            A = P @ vv.abs() + inner * (vis.double() @ vv.abs())
            to = u * o.abs() + tiny + (u + kappa) * A
            out["o"][0][b, :, h], out["o"][1][b, :, h] = o, to
            lse = torch.where(some, top + torch.log(torch.where(some, l, 1.0)), -math.inf)
            out["lse"][0][b, h], out["lse"][1][b, h] = lse, kappa + 4 * E * torch.where(some, lse, 0.0).abs()
            if do is None:
                continue
            g = torch.where(some[:, None], do[b, :, h], 0.0)
            dP, delta = g @ vv.T, (g * o).sum(1, keepdim=True)
            dS = torch.where(vis, P * (dP - delta) * fac, 0.0)
            edp = (D + 8) * E * (g.abs() @ vv.abs().T) + (g.abs() * (to + (D + 8) * E * o.abs())).sum(1, keepdim=True)
            eds = torch.where(vis, P * ((u + kappa + 16 * E) * (dP - delta).abs() * fac + edp * fac
                                        + (dP - delta).abs() * 8 * (float(dscore) / max(softcap, 1e-9) + E if softcap else 0.0)) + inner, 0.0)
            dq = dS @ kk * scale
            out["dq"][0][b, :, h] = dq
            out["dq"][1][b, :, h] = u * dq.abs() + tiny + scale * (eds @ kk.abs() + Sk * E * (dS.abs() @ kk.abs()))
            out["dk"][0][b, :, c] += dS.T @ qq * scale
            out["dk"][1][b, :, c] += scale * (eds.T @ qq.abs() + (Sq * H // Hk) * E * (dS.abs().T @ qq.abs()))
            out["dv"][0][b, :, c] += P.T @ g
            out["dv"][1][b, :, c] += (u + kappa + (Sq * H // Hk) * E) * (P.T @ g.abs()) + inner * (vis.double().T @ g.abs())
    for n in ("dk", "dv") if do is not None else ():
        out[n][1] += u * out[n][0].abs() + tiny
    return out


def _attention(type, B, Sq, Sk, H, Hk, D, seed=0, train=False, causal=False, softcap=0.0, slopes=False, k_lens=None, prefix=None,
               docs=None, scale=None, spoil=None, layout="plain"):
    import torch
    from paper_2206_08720_amd import seq
    q, k, v = (_rand(s, seed + n, type) for n, s in enumerate(((B, Sq, H, D), (B, Sk, Hk, D), (B, Sk, Hk, D))))
    do = _rand((B, Sq, H, D), seed + 3, type) if train else None
    opt = {"causal": causal, "softcap": softcap, "scale": scale,
           "slopes": torch.tensor([2.0 ** (-8 * (h + 1) / H) for h in range(H)]) if slopes else None,
           "k_lens": None if k_lens is None else torch.tensor(k_lens, dtype=torch.int32),
           "prefix": None if prefix is None else torch.tensor(prefix, dtype=torch.int32),
           "docs": None if docs is None else torch.tensor(docs, dtype=torch.int32).view(B, Sk)}
    if spoil:
        spoil(q, k, v, do)
    ref = _oracle(q, k, v, type, do, **opt)

    def place(t):
        if t is None:
            return None
        t = t.cuda()
        if layout == "heads_first":          # [batch, head, position, dim] in memory
            return t.transpose(1, 2).contiguous().transpose(1, 2)
        if layout == "odd":                  # rows of an odd stride at an odd place
            w = torch.zeros(t.shape[0], t.shape[1], t.shape[2], t.shape[3] + 3, dtype=t.dtype, device="cuda")
            w[..., 1:1 + t.shape[3]] = t
            return w[..., 1:1 + t.shape[3]]
        return t

    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in opt.items()}
    q, k, v, do = place(q), place(k), place(v), place(do)
    o, lse = seq.attention(q, k, v, return_lse=True, **dev)
    got = {"o": o, "lse": lse}
    if train:
        got["dq"], got["dk"], got["dv"] = seq.attention_backward(do, q, k, v, o, lse, **dev)
    torch.cuda.synchronize()
    for n, t in got.items():
        _close(n, t, *ref[n])
    return got


FORWARD = [
    # type, B, Sq, Sk, H, Hk, D, options
    ("bf16", 1, 1, 1, 1, 1, 64, {}),
    ("bf16", 2, 1, 777, 8, 8, 64, {"k_lens": [777, 300]}),
    ("f16", 3, 1, 1030, 8, 2, 128, {"k_lens": [1030, 1, 0], "causal": True}),
    ("f32", 2, 1, 515, 6, 3, 128, {"k_lens": [33, 515], "slopes": True}),
    ("bf16", 2, 5, 600, 12, 2, 80, {"k_lens": [600, 3], "causal": True, "softcap": 20.0}),
    ("bf16", 1, 7, 300, 4, 1, 96, {"causal": True, "docs": [j // 70 for j in range(300)]}),
    ("bf16", 1, 64, 64, 2, 2, 64, {"causal": True}),
    ("bf16", 2, 200, 200, 4, 2, 128, {}),
    ("f16", 1, 333, 333, 3, 1, 72, {"causal": True, "softcap": 30.0, "slopes": True}),
    ("f16", 2, 130, 517, 2, 1, 128, {"causal": True, "k_lens": [517, 60], "prefix": [100, 50]}),
    ("f32", 1, 161, 161, 2, 1, 40, {"causal": True, "prefix": [65]}),
    ("f32", 1, 96, 700, 2, 2, 128, {"causal": True, "softcap": 15.0}),
    ("bf16", 1, 300, 300, 2, 1, 64, {"causal": True, "docs": [-1] * 5 + [j // 64 for j in range(250)] + [9] * 30 + [-1] * 15}),
    ("bf16", 1, 70, 9000, 1, 1, 128, {"docs": [(j * 7919) % 50 for j in range(9000)]}),
    ("bf16", 1, 100, 100, 2, 1, 37, {"causal": True}),
    ("f16", 1, 65, 65, 1, 1, 1, {}),
    ("f32", 1, 50, 50, 2, 1, 3, {"causal": True, "scale": 0.7}),
]


@pytest.mark.parametrize("case", FORWARD, ids=lambda c: f"{c[0]}-{c[2]}x{c[3]}-{c[4]}.{c[5]}.{c[6]}-{'.'.join(c[7])}")
def test_attention_forward(case):
    _attention(*case[:7], seed=100, **case[7])


TRAIN = [
    ("f32", 1, 1, 1, 1, 1, 64, {}),
    ("f32", 2, 131, 131, 4, 2, 64, {"causal": True}),
    ("f32", 1, 97, 97, 2, 1, 128, {"causal": True, "prefix": [30], "slopes": True}),
    ("f32", 1, 61, 130, 2, 2, 48, {"causal": True, "softcap": 5.0, "k_lens": [100]}),
    ("bf16", 2, 300, 300, 4, 2, 128, {"causal": True}),
    ("bf16", 1, 200, 200, 6, 2, 64, {"causal": True, "docs": [j // 33 for j in range(180)] + [-1] * 20}),
    ("bf16", 2, 129, 129, 2, 1, 80, {"softcap": 10.0, "slopes": True}),
    ("f16", 1, 257, 257, 2, 2, 128, {"causal": True, "softcap": 30.0}),
    ("f16", 2, 40, 260, 4, 1, 96, {"causal": True, "k_lens": [260, 21], "prefix": [0, 200]}),
    ("bf16", 1, 77, 77, 2, 1, 45, {"causal": True}),
]


@pytest.mark.parametrize("case", TRAIN, ids=lambda c: f"{c[0]}-{c[2]}x{c[3]}-{c[4]}.{c[5]}.{c[6]}-{'.'.join(c[7])}")
def test_attention_backward(case):
    _attention(*case[:7], seed=200, train=True, **case[7])


@pytest.mark.parametrize("layout", ["heads_first", "odd"])
@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_attention_layouts(layout, type):
    _attention(type, 2, 70, 150, 4, 2, 64, seed=300, train=True, causal=True, layout=layout)
    _attention(type, 2, 1, 150, 4, 2, 64, seed=310, layout=layout)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_hidden_values_do_not_spread(value):
    """Values that are not finite where a mask hides them: an unfilled cache, padding, another document, the future."""
    def cache(q, k, v, do):
        k[0, 40:], v[0, 40:] = value, value

    _attention("bf16", 2, 1, 200, 4, 2, 64, seed=400, k_lens=[40, 200], spoil=cache)
    _attention("f32", 2, 40, 200, 4, 2, 64, seed=410, causal=True, k_lens=[40, 200], spoil=cache, train=True)

    def padding(q, k, v, do):
        for t in (q, k, v, do):
            t[0, 150:] = value

    docs = [j // 60 for j in range(150)] + [-1] * 50
    _attention("bf16", 1, 200, 200, 2, 1, 128, seed=420, causal=True, docs=docs, spoil=padding, train=True)


@pytest.mark.parametrize("type", ["bf16", "f16", "f32"])
def test_other_documents_values_do_not_spread(type):
    """One document is not finite: its own rows are not, every other result is that of the finite documents alone."""
    import torch
    from paper_2206_08720_amd import seq
    n, D = 160, 64
    docs = torch.tensor([j // 40 for j in range(n)], dtype=torch.int32)[None]
    q, k, v, do = (_rand((1, n, 2, D), 430 + i, type) for i in range(4))
    whole = _oracle(q, k, v, type, do, causal=True, docs=docs)
    k[0, 50, 0, 3], v[0, 60, 1, 7], v[0, 70, 0, 5] = math.nan, math.inf, math.nan
    o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), causal=True, docs=docs.cuda(), return_lse=True)
    grads = seq.attention_backward(do.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse, causal=True, docs=docs.cuda())
    keep = [i for i in range(n) if not 40 <= i < 80]
    for name, t in zip(("o", "dq", "dk", "dv"), (o,) + grads):
        _close(name, t[:, keep], whole[name][0][:, keep], whole[name][1][:, keep])
    o = o.cpu()
    assert torch.isfinite(o[0, 40:50]).all() and torch.isnan(o[0, 50:80, 0]).all()
    assert torch.isinf(o[0, 60:80, 1, 7]).all() and torch.isfinite(o[0, 60:80, 1, :7]).all()


@pytest.mark.parametrize("seed", range(60))
def test_random_attention(seed):
    """Random types, sizes, head groups, lengths, masks and layouts, forward and backward."""
    import random
    rng = random.Random(9000 + seed)
    type = rng.choice(("bf16", "f16", "f32"))
    B, Hk, G = rng.choice((1, 1, 2, 3)), rng.choice((1, 2, 3)), rng.choice((1, 2, 3, 5, 8))
    D = rng.choice((64, 128, rng.randrange(1, 129), 8 * rng.randrange(1, 17)))
    Sk = rng.choice((1, rng.randrange(2, 40), rng.randrange(40, 400), 64 * rng.randrange(1, 6)))
    Sq = rng.choice((1, Sk, Sk, rng.randrange(1, Sk + 1), min(Sk + 3, 50)))
    causal = rng.random() < 0.6
    opt = {"causal": causal, "softcap": rng.choice((0.0, 0.0, 3.0, 30.0)), "slopes": rng.random() < 0.3,
           "scale": rng.choice((None, None, 0.01, 0.6)), "layout": rng.choice(("plain", "plain", "heads_first", "odd"))}
    if rng.random() < 0.4:
        opt["k_lens"] = [rng.choice((0, 1, Sk, rng.randrange(Sk + 1))) for _ in range(B)]
    if causal and rng.random() < 0.3:
        opt["prefix"] = [rng.randrange(Sk + 1) for _ in range(B)]
    if rng.random() < 0.4:
        opt["docs"] = [rng.choice((-1, 0, 0, 1, 2)) if rng.random() < 0.1 else j // rng.choice((20, 70)) for _ in range(B) for j in range(Sk)]
    _attention(type, B, Sq, Sk, G * Hk, Hk, D, seed=9100 + 7 * seed, train=rng.random() < 0.7, **opt)


def test_attention_rows_that_see_nothing():
    import torch
    got = _attention("bf16", 2, 8, 20, 2, 1, 64, seed=440, train=True, causal=True, k_lens=[3, 0])
    assert not got["o"][0, :5].any() and not got["o"][1].any() and torch.isneginf(got["lse"][1]).all()
    assert not got["dq"][1].any() and not got["dk"][1].any() and not got["dk"][0, 3:].any()


@pytest.mark.parametrize("std", [2.0 ** -10, 2.0 ** 9])
def test_fp16_gradients_of_any_size(std):
    """Rows of 2000 keys: p and ds lie far below fp16's 2^-14, or above 2^15 with a large gradient; the backward pass scales
    them, so that no absolute step of theirs enters (o's does: the forward pass takes p as it is)."""
    import torch
    from paper_2206_08720_amd import seq
    q, k, v = (_rand((1, n, 1, 64), 530 + i, "f16") for i, n in enumerate((70, 2000, 2000)))
    do = _rand((1, 70, 1, 64), 533, "f16", std)
    o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), return_lse=True)
    grads = seq.attention_backward(do.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse)
    ref = _oracle(q, k, v, "f16", do, inner=0.0)
    loose = _oracle(q, k, v, "f16", do)
    _close("o", o, *loose["o"])
    # delta is formed from the stored o: its step there, times |dout|, enters ds through p
    extra = float((loose["o"][1] - ref["o"][1]).max()) * float(do.double().abs().sum(-1).max())
    P = torch.softmax(q[0, :, 0].double() @ k[0, :, 0].double().T / 8, 1)
    more = {"dq": extra / 8 * (P @ k[0, :, 0].double().abs())[None, :, None], "dk": extra / 8 * (P.T @ q[0, :, 0].double().abs())[None, :, None], "dv": 0.0}
    for name, g in zip(("dq", "dk", "dv"), grads):
        _close(name, g, ref[name][0], ref[name][1] + more[name])


def test_attention_gradient_against_differences():
    """The directional derivative of sum(w o) in 64 bits by central differences, against the gradients."""
    import torch
    from paper_2206_08720_amd import seq
    q, k, v, w = (_rand(s, 500 + i, "f32") for i, s in enumerate(((1, 37, 4, 32), (1, 50, 2, 32), (1, 50, 2, 32), (1, 37, 4, 32))))
    opt = {"causal": True, "softcap": 4.0, "slopes": torch.tensor([0.1, 0.05, 0.02, 0.01]), "prefix": torch.tensor([9], dtype=torch.int32)}
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in opt.items()}
    o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), return_lse=True, **dev)
    grads = seq.attention_backward(w.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse, **dev)
    tol = _oracle(q, k, v, "f32", w, **opt)
    x = [t.double() for t in (q, k, v)]
    for i, (name, g) in enumerate(zip(("dq", "dk", "dv"), grads)):
        d = _rand(x[i].shape, 510 + i).double()
        f = [(_oracle(*[t + (s * 1e-4 * d if n == i else 0) for n, t in enumerate(x)], "f32", **opt)["o"][0] * w.double()).sum() for s in (1, -1)]
        diff = (f[0] - f[1]) / 2e-4
        # the quotient's own error: 1e-8 of third derivatives of order one a term
        assert abs(float((g.cpu().double() * d).sum() - diff)) <= float((tol[name][1] * d.abs()).sum()) + 1e-6 * float(d.abs().sum()), name


def test_attention_offsets_past_32_bits():
    """A cache whose last keys lie over 4 GiB into it (and past 2^31 elements)."""
    import torch
    from paper_2206_08720_amd import seq
    n, hk, D = 300, 2, 128
    big = torch.empty((n * 30000 * 2 * D,), dtype=torch.bfloat16, device="cuda")
    k = big.view(1, n, 30000 * 2, D)[:, :, :hk]
    v = big.view(1, n, 30000 * 2, D)[:, :, hk:2 * hk]
    kc, vc, q = _rand((1, n, hk, D), 521, "bf16"), _rand((1, n, hk, D), 522, "bf16"), _rand((1, 1, 4, D), 523, "bf16")
    k.copy_(kc)
    v.copy_(vc)
    ref = _oracle(q, kc, vc, "bf16")
    _close("o", seq.attention(q.cuda(), k, v), *ref["o"])
    q2 = _rand((1, 200, 4, D), 524, "bf16")
    _close("o", seq.attention(q2.cuda(), k, v, causal=True), *_oracle(q2, kc, vc, "bf16", causal=True)["o"])


def test_many_documents_in_long_rows():
    """More tiles than the lists of a workgroup hold (2^14 tiles of 32 rows; of 32 and of 64 keys): what lies past them is
    left to the masks."""
    import torch
    from paper_2206_08720_amd import seq
    n, D, doc = 530000, 64, 90
    docs = (torch.arange(n) // doc).int()
    q, k, v, do = (torch.randn(1, n, 1, D, generator=torch.Generator("cuda").manual_seed(540 + i), device="cuda").bfloat16() for i in range(4))
    opt = {"causal": True, "docs": docs[None].cuda()}
    o, lse = seq.attention(q, k, v, return_lse=True, **opt)
    grads = seq.attention_backward(do, q, k, v, o, lse, **opt)
    last = n - (n - 1) // doc * doc
    for a, b in ((0, 2 * doc), (262080, 262080 + doc), (n - last - doc, n)):   # whole documents
        part = [t[:, a:b].cpu() for t in (q, k, v)]
        ref = _oracle(*part, "bf16", do[:, a:b].cpu(), causal=True, docs=docs[None, a:b])
        for name, t in zip(("o", "dq", "dk", "dv"), (o,) + grads):
            _close(f"{name} {a}", t[:, a:b], *ref[name])
    # one token, and a few rows, over two copies of the keys
    ids = torch.cat((docs, docs + docs[-1] + 1))
    far = {"docs": ids[None].cuda()}
    k2, v2 = torch.cat((k, k), 1), torch.cat((v, v), 1)
    for rows in (1, 40):
        a = n - last
        ref = _oracle(q[:, n - rows:].cpu(), k[:, a:].cpu(), v[:, a:].cpu(), "bf16", docs=docs[None, a:])
        _close(f"o {rows}", seq.attention(q[:, n - rows:], k2, v2, **far), *ref["o"])


# ---- norm -----------------------------------------------------------------------------------------------------------

def _norm_reference(x, res, w, eps, type, dy=None, dh=None, h_saved=None):
    import torch
    u, tiny, n = U[type], TINY[type], x.shape[-1]
    x, w = x.double(), w.double()
    h = x + (0 if res is None else res.double())
    r = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    y = h * r * w
    rel = (n + 8) * E
    out = {"y": (y, (u + rel) * y.abs() + tiny), "h": (h, (u + 2 * E) * h.abs() + tiny)}
    if dy is not None:
        h = h_saved.double()
        r = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
        g = dy.double() * w
        m = (g * h).mean(-1, keepdim=True)
        e = dh.double() if dh is not None else torch.zeros_like(h)
        dx = r * (g - h * r * r * m) + e
        mag = r * (g.abs() + h.abs() * r * r * (g * h).abs().mean(-1, keepdim=True)) + e.abs()
        out["dx"] = (dx, u * dx.abs() + tiny + 4 * rel * mag)
        t = dy.double() * h * r
        dw = t.sum(0)
        out["dw"] = (dw, u * dw.abs() + tiny + (rel + (x.shape[0] + 8) * E) * t.abs().sum(0))
    return out


NORM = [(type, rows, n) for type in ("bf16", "f16", "f32")
        for rows, n in ((1, 1), (3, 7), (5, 512), (9, 785), (130, 1000), (4, 1024), (17, 2048), (6, 4096), (1100, 96), (3, 8192), (2, 12289), (2, 32768))]


@pytest.mark.parametrize("type,rows,n", NORM)
def test_rms_norm(type, rows, n):
    import torch
    from paper_2206_08720_amd import seq
    x, res, dy, dh = (_rand((rows, n), 600 + i, type, s) for i, s in enumerate((1.0, 3.0, 1.0, 0.5)))
    for wtype in dict.fromkeys((type, "f32")):
        w = (1 + 0.1 * _rand((n,), 610)).to(_types()[wtype])
        y, h = seq.rms_norm(x.cuda(), w.cuda(), residual=res.cuda(), eps=1e-5)
        ref = _norm_reference(x, res, w, 1e-5, type, dy, dh, h.cpu())
        _close("y", y, *ref["y"])
        _close("h", h, *ref["h"])
        dx, dw = seq.rms_norm_backward(dy.cuda(), h, w.cuda(), dh=dh.cuda(), eps=1e-5)
        _close("dx", dx, *ref["dx"])
        val, tol = ref["dw"]
        assert dw.dtype == w.dtype
        _close("dw", dw, val, tol - U[type] * val.abs() + U[wtype] * val.abs())
    y = seq.rms_norm(x.cuda(), w.cuda())
    _close("y", y, *_norm_reference(x, None, w, 1e-6, type)["y"])


def test_rms_norm_e4m3_of_tiny_rows():
    """max|y| / 448 below the smallest normal fp32: the scale stays at it and nothing turns into NaN."""
    import torch
    from paper_2206_08720_amd import seq
    x = torch.zeros(1, 64, device="cuda")
    x[0, 3] = 1.0
    q, scale = seq.rms_norm_e4m3(x, torch.full((64,), 1e-43, device="cuda"))
    assert float(scale) == 2.0 ** -126 and torch.isfinite(q.float()).all()


@pytest.mark.parametrize("type,rows,n", [("bf16", 5, 2048), ("f16", 3, 777), ("f32", 2, 20000), ("bf16", 1, 1)])
def test_rms_norm_e4m3(type, rows, n):
    """q scale is y within half a step of e4m3 (2^-4 of the value, or 2^-10 of the scale near zero)."""
    import torch
    from paper_2206_08720_amd import seq
    x, res, w = _rand((rows, n), 620, type, 2.0), _rand((rows, n), 621, type), (1 + 0.1 * _rand((n,), 622)).to(_types()[type])
    x[0], res[0] = 0, 0                                  # a row of zeros
    q, scale, h = seq.rms_norm_e4m3(x.cuda(), w.cuda(), residual=res.cuda())
    y, tol = _norm_reference(x, res, w, 1e-6, "f32")["y"]
    assert q.dtype == torch.float8_e4m3fn and float(scale[0]) == 1.0
    most = y.abs().max(1).values
    _close("scale", scale[1:], (most / 448)[1:], ((n + 16) * E * most)[1:])
    s = scale.cpu().double()[:, None]
    _close("q", q.float().cpu() * scale.cpu()[:, None], y, 2 * tol + torch.maximum(y.abs() / 16, s * 2.0 ** -10) * (1 + 1e-3))
    _close("h", h, *_norm_reference(x, res, w, 1e-6, type)["h"])


def test_rms_norm_strides_and_values_in_place():
    import torch
    from paper_2206_08720_amd import seq
    wide = _rand((40, 3000), 630, "bf16").cuda()
    w = torch.ones(1001, dtype=torch.bfloat16, device="cuda")
    for lo in (0, 8, 13):
        x = wide[:, lo:lo + 1001]
        _close("y", seq.rms_norm(x, w), *_norm_reference(x.cpu(), None, w.cpu(), 1e-6, "bf16")["y"])
    one = _rand((1, 1, 64), 631, "bf16").cuda()
    y, h = seq.rms_norm(one.expand(5, 3, 64), w[:64].clone(), residual=one.expand(5, 3, 64))    # broadcast rows
    assert torch.equal(y[4, 2], y[0, 0]) and torch.equal(h[4, 2], 2 * one[0, 0])
    x = wide[:3, :64].clone()
    x[1, 5] = math.nan
    y = seq.rms_norm(x, w[:64].clone())
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()


def test_rms_norm_gradient_against_differences():
    import torch
    from paper_2206_08720_amd import seq
    x, res, w, c, dh = _rand((5, 33), 640), _rand((5, 33), 641), 1 + 0.1 * _rand((33,), 642), _rand((5, 33), 643), _rand((5, 33), 644)
    y, h = seq.rms_norm(x.cuda(), w.cuda(), residual=res.cuda())
    dx, dw = seq.rms_norm_backward(c.cuda(), h, w.cuda(), dh=dh.cuda())
    tol = _norm_reference(x, res, w, 1e-6, "f32", c, dh, h.cpu())

    def loss(x, w):
        r = _norm_reference(x, res, w, 1e-6, "f32")
        return float((r["y"][0] * c.double()).sum() + (r["h"][0] * dh.double()).sum())

    d = _rand(x.shape, 645).double()
    diff = (loss(x.double() + 1e-4 * d, w) - loss(x.double() - 1e-4 * d, w)) / 2e-4
    assert abs(float((dx.cpu().double() * d).sum()) - diff) <= float((tol["dx"][1] * d.abs()).sum()) + 1e-6 * float(d.abs().sum())
    d = _rand(w.shape, 646).double()
    diff = (loss(x, w.double() + 1e-4 * d) - loss(x, w.double() - 1e-4 * d)) / 2e-4
    assert abs(float((dw.cpu().double() * d).sum()) - diff) <= float((tol["dw"][1] * d.abs()).sum()) + 1e-6 * float(d.abs().sum())


# ---- rotary ---------------------------------------------------------------------------------------------------------

def _table(max_pos, rot, base=10000.0, kind=None, factor=1.0, original=0, low=1.0, high=32.0):
    import torch
    j = torch.arange(0, rot, 2, dtype=torch.float64)
    if kind == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-j / rot)
    mag = 1.0
    if kind == "linear":
        f = f / factor
    if kind == "ramp":
        keep = ((f * original / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f, mag = f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1
    a = torch.arange(max_pos, dtype=torch.float64)[:, None] * f
    return torch.stack((a.cos(), a.sin()), -1) * mag


@pytest.mark.parametrize("kind", [None, "linear", "base", "ramp"])
def test_rotary_table(kind):
    from paper_2206_08720_amd import seq
    n, rot = 150000, 64
    got = seq.rotary_table(n, rot, base=500000.0, scaling=kind, factor=8.0, original=8192)
    ref = _table(n, rot, 500000.0, kind, 8.0, 8192)
    # 64-bit angles of up to 1.5e5 and their frequencies' few roundings: 1e-10; one rounding to fp32
    _close("table", got, ref, 2.0 ** -24 * ref.abs() + 2.0 ** -25 + 1e-9)


def _rotary_reference(x, table, at, interleaved, inverse):
    import torch
    rot = 2 * table.shape[1]
    t = table.double()[at.long()]
    c, s = t[..., 0][:, :, None], t[..., 1][:, :, None] * (-1 if inverse else 1)
    x = x.double()
    u, v = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b, mag = u * c - v * s, v * c + u * s, u.abs() * c.abs() + v.abs() * s.abs() + v.abs() * c.abs() + u.abs() * s.abs()
    out, m = x.clone(), torch.zeros_like(x)
    if interleaved:
        out[..., 0:rot:2], out[..., 1:rot:2], m[..., 0:rot:2], m[..., 1:rot:2] = a, b, mag, mag
    else:
        out[..., :rot // 2], out[..., rot // 2:rot], m[..., :rot // 2], m[..., rot // 2:rot] = a, b, mag, mag
    return out, m


@pytest.mark.parametrize("type,B,n,H,Hk,D,rot,interleaved", [
    ("bf16", 2, 33, 4, 2, 128, 128, False), ("bf16", 1, 1, 8, 1, 64, 64, True), ("f16", 3, 7, 3, 3, 80, 32, True),
    ("f32", 2, 17, 2, 1, 96, 48, False), ("f32", 1, 5, 1, 1, 10, 6, False), ("f16", 2, 9, 2, 1, 37, 14, True),
    ("bf16", 1, 300, 16, 4, 128, 64, False)])
def test_rotary(type, B, n, H, Hk, D, rot, interleaved):
    import torch
    from paper_2206_08720_amd import seq
    table = _table(500, rot).float()
    q, k = _rand((B, n, H, D), 700, type), _rand((B, n, Hk, D), 701, type)
    at = torch.randint(0, 500, (B, n), generator=torch.Generator().manual_seed(702), dtype=torch.int32)
    for inverse in (False, True):
        a, b = seq.rotary(q.cuda(), table.cuda(), at.cuda(), k=k.cuda(), interleaved=interleaved, inverse=inverse)
        for name, x, y in (("q", q, a), ("k", k, b)):
            ref, mag = _rotary_reference(x, table, at, interleaved, inverse)
            _close(name, y, ref, U[type] * ref.abs() + TINY[type] + 3 * E * mag)
    # in place, in a packed projection, positions from a first one
    packed = torch.cat((q, k, k), 2).cuda()
    qv, kv, rest = packed.split((H, Hk, Hk), 2)
    seq.rotary(qv, table.cuda(), 11, k=kv, interleaved=interleaved, inplace=True)
    run = 11 + torch.arange(n).expand(B, n)
    for name, x, y in (("q", q, qv), ("k", k, kv)):
        ref, mag = _rotary_reference(x, table, run, interleaved, False)
        _close(name, y, ref, U[type] * ref.abs() + TINY[type] + 3 * E * mag)
    assert torch.equal(rest.cpu(), k)


def test_rotary_positions_outside_the_table_are_nan():
    import torch
    from paper_2206_08720_amd import seq
    q = _rand((1, 4, 2, 64), 710, "bf16").cuda()
    y = seq.rotary(q, seq.rotary_table(10, 64), torch.tensor([[3, -1, 10, 9]], dtype=torch.int32, device="cuda"))
    assert torch.isnan(y[0, 1:3]).all() and torch.isfinite(y[0, [0, 3]]).all()


# ---- streams, graphs, refusals --------------------------------------------------------------------------------------

def test_other_stream_and_determinism():
    import torch
    from paper_2206_08720_amd import seq
    q, k, v = (_rand((2, 90, h, 64), 800 + h, "bf16").cuda() for h in (4, 2, 2))
    one = seq.attention(q, k, v, causal=True, return_lse=True)
    g1 = seq.attention_backward(q, q, k, v, *one, causal=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    two = seq.attention(q, k, v, causal=True, return_lse=True, stream=s)
    g2 = seq.attention_backward(q, q, k, v, *two, causal=True, stream=s)
    s.synchronize()
    for a, b in zip(one + g1, two + g2):
        assert torch.equal(a, b)


def test_graph_replay_matches_eager():
    import torch
    from paper_2206_08720_amd import seq
    x, w = _rand((6, 512), 810, "bf16").cuda(), torch.ones(512, dtype=torch.bfloat16, device="cuda")
    cache = _rand((6, 900, 2, 2, 64), 811, "bf16").cuda()
    table = seq.rotary_table(1000, 64)
    lens = torch.tensor([900, 1, 40, 899, 500, 0], dtype=torch.int32, device="cuda")

    def step():
        y, h = seq.rms_norm(x, w, residual=x)
        q = seq.rotary(y.view(6, 1, 8, 64), table, 5)
        o, lse = seq.attention(q, cache[:, :, 0], cache[:, :, 1], k_lens=lens, return_lse=True)
        dq, dk, dv = seq.attention_backward(q, q, cache[:, :, 0], cache[:, :, 1], o, lse, k_lens=lens)
        dx, dw = seq.rms_norm_backward(dq.view(6, 512), h, w)
        return o, dq, dk, dv, dx, dw

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(_rand((6, 512), 820 + k, "bf16"))
        lens.copy_(torch.tensor([900 - k, 1 + k, 40, 899, 500, k], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b)


def test_refusals():
    import torch
    from paper_2206_08720_amd import _lib, seq
    q, k = torch.zeros(1, 4, 4, 64, device="cuda"), torch.zeros(1, 4, 2, 64, device="cuda")
    ids = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        seq.attention(q.cpu(), k, k)
    with pytest.raises(TypeError):
        seq.attention(q, k.half(), k.half())
    with pytest.raises(ValueError):
        seq.attention(q, k, k[:, :3])
    with pytest.raises(ValueError):
        seq.attention(q.transpose(2, 3), k, k)
    with pytest.raises(TypeError):
        seq.attention(q, k, k, docs=ids.long())
    for bad, code in (({"softcap": -1.0}, _lib.NTK_E_ARG), ({"softcap": math.nan}, _lib.NTK_E_ARG), ({"scale": 0.0}, _lib.NTK_E_ARG),
                      ({"prefix": ids[0, :1].clone()}, _lib.NTK_E_ARG)):
        with pytest.raises(_lib.NTKError) as e:
            seq.attention(q, k, k, **bad)
        assert e.value.code == code
    with pytest.raises(_lib.NTKError) as e:
        seq.attention(q[:, :, :3], k, k)
    assert e.value.code == _lib.NTK_E_SHAPE
    wide = torch.zeros(1, 4, 2, 136, device="cuda")
    with pytest.raises(_lib.NTKError) as e:
        seq.attention(wide, wide, wide)
    assert e.value.code == _lib.NTK_E_UNSUPPORTED
    with pytest.raises(_lib.NTKError) as e:
        seq.rms_norm(torch.zeros(1, 32769, device="cuda"), torch.zeros(32769, device="cuda"))
    assert e.value.code == _lib.NTK_E_UNSUPPORTED
    with pytest.raises(ValueError):
        seq.rms_norm(q, torch.zeros(63, device="cuda"))
    for weight in (None, torch.zeros(64, device="cuda").half(), torch.zeros(64)):
        with pytest.raises(TypeError):
            seq.rms_norm(q, weight)
        with pytest.raises(TypeError):
            seq.rms_norm_backward(q, q, weight)
    with pytest.raises(_lib.NTKError) as e:
        seq.rotary(q, seq.rotary_table(8, 66))
    assert e.value.code == _lib.NTK_E_SHAPE
    with pytest.raises(ValueError):
        seq.rotary_table(8, 63)


def test_empty_sizes():
    import torch
    from paper_2206_08720_amd import seq
    for B, Sq, Sk in ((0, 4, 4), (2, 0, 5), (2, 4, 0)):
        q, k = torch.ones(B, Sq, 2, 64, device="cuda"), torch.ones(B, Sk, 1, 64, device="cuda")
        o, lse = seq.attention(q, k, k, return_lse=True)
        grads = seq.attention_backward(q, q, k, k, o, lse)
        torch.cuda.synchronize()
        assert not o.any() and torch.isneginf(lse).all() and not any(g.any() for g in grads)
    x, w = torch.ones(0, 64, device="cuda"), torch.ones(64, device="cuda")
    assert seq.rms_norm(x, w).shape == (0, 64)
    dx, dw = seq.rms_norm_backward(x, x, w)
    assert dx.shape == (0, 64) and not dw.any()
    assert seq.rotary(torch.ones(2, 0, 3, 64, device="cuda"), seq.rotary_table(4, 64)).shape == (2, 0, 3, 64)
