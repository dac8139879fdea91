"""Values at the edge of the sequence operators' ranges (paper_2206_08720_amd.seq): weights far below the largest, operands that
are not finite, saturated scores, rows of extreme size.  The tolerances are those of tests/test_gpu_seq.py, whose
definitions in 64 bits are used here too, or derived beside a test.
"""
import math

import pytest

from tests.test_gpu_seq import E, TINY, U, _attention, _close, _norm_reference, _oracle, _rand, _types

pytestmark = pytest.mark.gpu


# ---- fp16 weights far below the largest -----------------------------------------------------------------------------

@pytest.mark.parametrize("gap", [15.0, 17.0, 17.5])
@pytest.mark.parametrize("rows,keys,heads", [(1, 32768, 1), (40, 6000, 1), (33, 2000, 192)])
def test_fp16_weights_far_below_the_largest(rows, keys, heads, gap):
    """One key with v = 0 takes nearly all the weight, and thousands of others share what is left.  The forward pass forms weights times
    2^14, so that half a smallest step of them is 2^-25 2^-14.  One token and its ranges, row tiles in ranges and whole."""
    import torch
    from paper_2206_08720_amd import seq
    q, k = torch.zeros(1, rows, heads, 64).half(), torch.zeros(1, keys, heads, 64).half()
    v = (_rand((1, keys, heads, 64), 900).abs() + 0.5).half()
    q[..., 0], k[0, 77, :, 0], v[0, 77] = 8.0, gap, 0.0
    o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), return_lse=True)
    few = slice(0, 2)                                  # all heads are alike in what they go through
    ref = _oracle(q[:, :, few], k[:, :, few], v[:, :, few], "f16", inner=2.0 ** -39)
    _close("o", o[:, :, few], *ref["o"])
    _close("lse", lse[:, few], *ref["lse"])


def test_fp16_gradient_of_values_of_small_weight():
    """Weights of 2^-33, whose sum over the rows with large gradients is dv: formed times 2^14 too.  (The heavy key's own dv is past fp16's
    largest.)"""
    import torch
    from paper_2206_08720_amd import seq
    q, k, v = torch.zeros(1, 64, 1, 64).half(), torch.zeros(1, 300, 1, 64).half(), _rand((1, 300, 1, 64), 905, "f16")
    do = (1000 * (1 + _rand((1, 64, 1, 64), 906).abs())).half()
    q[..., 0], k[0, 77, :, 0] = 8.0, 23.0
    o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), return_lse=True)
    dv = seq.attention_backward(do.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse)[2]
    keep = [j for j in range(300) if j != 77]
    ref, tol = _oracle(q, k, v, "f16", do, inner=2.0 ** -39)["dv"]
    _close("dv", dv[:, keep], ref[:, keep], tol[:, keep])


# ---- infinities -----------------------------------------------------------------------------------------------------

FORMS = [("f32", 1), ("f32", 64), ("bf16", 1), ("bf16", 64), ("f16", 64)]


@pytest.mark.parametrize("type,rows", FORMS)
def test_visible_key_at_minus_infinity(type, rows):
    """A key that is -inf where all queries are positive has scores of -inf and no weight: o, lse, dv and the other keys' dk are
    those without it, its own dk and dv are 0; dq meets 0 * inf in that component alone."""
    import torch
    from paper_2206_08720_amd import seq
    n, D, at, d = 150, 64, 70, 3
    q, k, v, do = (_rand((1, m, 2, D), 910 + i, type) for i, m in enumerate((rows, n, n, rows)))
    q[..., d] = q[..., d].abs() + 0.5
    keep = [j for j in range(n) if j != at]
    ref = _oracle(q, k[:, keep], v[:, keep], type, do)
    k[0, at, :, d] = -math.inf
    o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), return_lse=True)
    _close("o", o, *ref["o"])
    _close("lse", lse, *ref["lse"])
    if rows % 32:
        return
    dq, dk, dv = seq.attention_backward(do.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse)
    _close("dk", dk[:, keep], *ref["dk"])
    _close("dv", dv[:, keep], *ref["dv"])
    assert not dk[0, at].any() and not dv[0, at].any()
    rest = [c for c in range(D) if c != d]
    _close("dq", dq[..., rest], ref["dq"][0][..., rest], ref["dq"][1][..., rest])
    assert not torch.isfinite(dq[..., d]).any()


@pytest.mark.parametrize("type,rows", FORMS)
def test_infinities_reach_what_meets_them(type, rows):
    """An infinite key: rows whose score is -inf do without it, those at +inf or 0 * inf are NaN.  An infinite query: its row alone.
    An infinite value or gradient of o: its component alone, with its sign."""
    import torch
    from paper_2206_08720_amd import seq
    n, D, at, d = 150, 64, 20, 5
    q, k, v = (_rand((1, m, 2, D), 920 + i, type) for i, m in enumerate((rows, n, n)))
    keep = [j for j in range(n) if j != at]
    q[0, -1, :, d] = 0.0
    for value in (math.inf, -math.inf):
        spoilt = k.clone()
        spoilt[0, at, :, d] = value
        out = seq.attention(q.cuda(), spoilt.cuda(), v.cuda()).cpu()
        without = (q[..., d].double() * value == -math.inf)[..., None].expand(out.shape)
        ref, tol = _oracle(q, k[:, keep], v[:, keep], type)["o"]
        _close("o", torch.where(without, out.double(), 0.0), torch.where(without, ref, 0.0), tol)
        assert torch.isnan(out[~without]).all()
        spoilt = v.clone()
        spoilt[0, at, :, d] = value
        out = seq.attention(q.cuda(), k.cuda(), spoilt.cuda()).cpu()
        ref, tol = _oracle(q, k, v, type)["o"]
        assert (out[..., d] == value).all()
        out[..., d], ref[..., d] = 0.0, 0.0
        _close("o", out, ref, tol)
        spoilt = q.clone()
        spoilt[0, 0, 0, d] = value
        out = seq.attention(spoilt.cuda(), k.cuda(), v.cuda()).cpu()
        ref, tol = _oracle(q, k, v, type)["o"]
        assert torch.isnan(out[0, 0, 0]).all()
        out[0, 0, 0], ref[0, 0, 0] = 0.0, 0.0
        _close("o", out, ref, tol)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
def test_infinite_gradient_reaches_its_component_of_dv(type):
    import torch
    from paper_2206_08720_amd import seq
    q, k, v, do = (_rand((1, m, 2, 64), 930 + i, type) for i, m in enumerate((64, 150, 150, 64)))
    ref, tol = _oracle(q, k, v, type, do)["dv"]
    do[0, 9, :, 5] = -math.inf
    o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), return_lse=True)
    dv = seq.attention_backward(do.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse)[2].cpu()
    assert (dv[..., 5] == -math.inf).all()
    dv[..., 5], ref[..., 5] = 0.0, 0.0
    _close("dv", dv, ref, tol)


@pytest.mark.parametrize("rows", [1, 64])
def test_nan_of_any_payload_stays_nan(rows):
    """fp32 NaN whose payload lies in the lowest bit, of either sign."""
    import torch
    from paper_2206_08720_amd import seq
    q, k, v = (_rand((1, m, 1, 64), 940 + i) for i, m in enumerate((rows, 150, 150)))
    q[..., 5] = q[..., 5].abs() + 0.5
    for bits in (0x7f800001, 0xff800001 - (1 << 32)):
        k[0, 20].view(torch.int32)[0, 5] = bits
        assert torch.isnan(seq.attention(q.cuda(), k.cuda(), v.cuda())).all()


@pytest.mark.parametrize("type,cap", [("f32", 0.0), ("bf16", 0.0), ("f16", 0.0), ("f32", 5.0), ("bf16", 5.0), ("f16", 5.0)])
def test_infinite_operand_against_a_weight_of_zero_is_nan(type, cap):
    """dq = ds k and dk = ds^T q: an infinite k or q that a pair sees has a score of -inf (weight 0), or with a cap a derivative of 0,
    so it is multiplied by 0 and gives NaN, whatever its sign."""
    import torch
    from paper_2206_08720_amd import seq
    for sign in (1.0, -1.0):
        q, k, v, do = (_rand((1, m, 1, 64), 945 + i, type) for i, m in enumerate((64, 150, 150, 64)))
        q[..., 3] = -sign * (q[..., 3].abs() + 0.5)
        k[0, 20, 0, 3] = sign * math.inf
        o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), softcap=cap, return_lse=True)
        dq, dk, _ = seq.attention_backward(do.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse, softcap=cap)
        assert torch.isnan(dq[..., 3]).all() and torch.isfinite(dq[..., :3]).all() and torch.isfinite(dk).all()
        if cap:                                        # the same with an infinite query: its scores are all +-cap
            q, k = _rand((1, 64, 1, 64), 945, type), _rand((1, 150, 1, 64), 946, type)
            q[0, 20, 0, 3] = sign * math.inf
            k[..., 3] = k[..., 3].abs() + 0.5
            o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), softcap=cap, return_lse=True)
            dq, dk, _ = seq.attention_backward(do.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse, softcap=cap)
            assert torch.isnan(dk[..., 3]).all() and torch.isfinite(dk[..., :3]).all() and torch.isfinite(dq).all()


# ---- heads dealt out to the dies ------------------------------------------------------------------------------------

def _spoil_tail(q, k, v, do):
    k[0, -40:], v[0, -40:] = math.nan, math.inf


EIGHTS = [
    # batch * kv_heads is 8 or 16: each die takes its own heads; several tiles and ranges a head
    ("bf16", 1, 300, 300, 8, 8, 64, {"causal": True, "train": True}),
    ("f32", 2, 300, 300, 8, 8, 64, {"causal": True, "train": True}),
    ("bf16", 2, 520, 520, 16, 8, 128, {"causal": True, "train": True}),
    ("f16", 4, 200, 390, 4, 2, 80, {"train": True, "softcap": 20.0}),
    ("f16", 2, 300, 300, 16, 4, 64, {"causal": True, "train": True, "docs": [j // 90 for _ in range(2) for j in range(300)]}),
    ("bf16", 2, 1, 4000, 16, 8, 128, {"k_lens": [4000, 1777]}),
    ("f32", 8, 3, 1200, 2, 1, 64, {"causal": True}),
    ("bf16", 2, 1, 4000, 8, 8, 64, {"k_lens": [3960, 4000], "spoil": _spoil_tail}),
    ("bf16", 2, 300, 300, 8, 4, 64, {"causal": True, "train": True, "k_lens": [260, 300], "spoil": _spoil_tail}),
    ("f32", 1, 200, 300, 8, 8, 128, {"train": True, "k_lens": [260], "spoil": _spoil_tail}),
]


@pytest.mark.parametrize("case", EIGHTS, ids=lambda c: f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-{c[4]}.{c[5]}.{c[6]}-{'.'.join(c[7])}")
def test_heads_in_eights(case):
    _attention(*case[:7], seed=950, **case[7])


@pytest.mark.parametrize("seed", range(12))
def test_random_attention_of_eight_heads(seed):
    import random
    rng = random.Random(9500 + seed)
    type, B, G = rng.choice(("bf16", "f16", "f32")), rng.choice((1, 2)), rng.choice((1, 2))
    Sk = rng.randrange(130, 420)
    opt = {"causal": rng.random() < 0.6, "softcap": rng.choice((0.0, 10.0)), "slopes": rng.random() < 0.3}
    if rng.random() < 0.4:
        opt["k_lens"] = [rng.randrange(Sk + 1) for _ in range(B)]
    _attention(type, B, rng.choice((2, Sk, Sk)), Sk, 8 * G, 8, rng.choice((40, 64, 128)), seed=9600 + 7 * seed, train=True, **opt)


# ---- row tiles that end past the rows -------------------------------------------------------------------------------

@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 50, 96])
def test_key_at_minus_infinity_with_odd_rows(type, rows):
    """As test_visible_key_at_minus_infinity, with the last tile of 32 rows partly empty: what is not a row meets no key."""
    from paper_2206_08720_amd import seq
    n, D, at, d = 150, 64, 70, 3
    q, k, v, do = (_rand((1, m, 1, D), 960 + i, type) for i, m in enumerate((rows, n, n, rows)))
    q[..., d] = q[..., d].abs() + 0.5
    keep = [j for j in range(n) if j != at]
    ref = _oracle(q, k[:, keep], v[:, keep], type, do)
    k[0, at, :, d] = -math.inf
    o, lse = seq.attention(q.cuda(), k.cuda(), v.cuda(), return_lse=True)
    _, dk, dv = seq.attention_backward(do.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse)
    _close("dk", dk[:, keep], *ref["dk"])
    _close("dv", dv[:, keep], *ref["dv"])
    assert not dk[0, at].any() and not dv[0, at].any()


def _one_head(type, q, k, v, do, scale, cap=0.0, bias=None):
    """{name: (value, tolerance)} for q, do [rows, D], k, v [n, D] that all see each other, in 64 bits.  The tolerances are those of
    _oracle, with a score's error taken from the magnitudes of its terms (the bias [rows, n] may have any sign), and with that of the cap's
    derivative taken relatively: 4 e / (1 + e)^2 with e = exp(-2 |y|), y = scale x / cap, changes by 2 |dy| and by
    6 roundings of y's factor, which are 12 |y| E < 120 E here.  Weights below 2^-126 may vanish."""
    import torch
    u, tiny, D, n = U[type], TINY[type], q.shape[1], k.shape[0]
    inner = 2.0 ** -35 if type == "f16" else 0.0         # fp16's p and ds are formed times 2^10 and more
    q, k, v, do = (t.double() for t in (q, k, v, do))
    x = q @ k.T * scale
    far = torch.zeros_like(x) if bias is None else bias.double()
    s = (cap * torch.tanh(x / cap) if cap else x) - far
    P, lse = torch.softmax(s, 1), torch.logsumexp(s, 1)
    dx = (D + 8) * E * float((q.abs() @ k.abs().T * scale + far.abs()).max())
    kappa = 2 * (dx + 8 * E * cap) + (n + 8) * E
    fac, rel = (1 / torch.cosh(x / cap) ** 2, 2 * dx / cap + 120 * E) if cap else (torch.ones_like(x), 0.0)
    o = P @ v
    least = 2.0 ** -126
    to = u * o.abs() + tiny + (u + kappa) * (P @ v.abs()) + least * v.abs().sum(0)
    dP, delta = do @ v.T, (do * o).sum(1, keepdim=True)
    dS = P * (dP - delta) * fac
    edp = (D + 8) * E * (do.abs() @ v.abs().T) + (do.abs() * (to + (D + 8) * E * o.abs())).sum(1, keepdim=True)
    eds = P * fac * ((u + kappa + 16 * E + rel) * (dP - delta).abs() + edp) + least * (dP - delta).abs() + inner
    out = {"o": (o, to), "lse": (lse, kappa + 4 * E * lse.abs())}
    for name, a, b, err, m in (("dq", dS, k, eds, n), ("dk", dS.T, q, eds.T, len(q))):
        g = a @ b * scale
        out[name] = (g, u * g.abs() + tiny + scale * (err @ b.abs() + m * E * (a.abs() @ b.abs())))
    dv = P.T @ do
    out["dv"] = (dv, u * dv.abs() + tiny + (u + kappa + len(q) * E) * (P.T @ do.abs()) + (inner + least) * do.abs().sum(0))
    return out


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [33, 64])
def test_slopes_that_favour_distance(type, rows):
    """Negative slopes: far keys weigh most, and e^(-slope distance) alone is not finite in 32 bits."""
    import torch
    from paper_2206_08720_amd import seq
    q, k, v, do = (_rand((m, 64), 970 + i, type) for i, m in enumerate((rows, 200, 200, rows)))
    far = (200 - rows + torch.arange(rows)[:, None] - torch.arange(200)).abs()
    ref = _one_head(type, q, k, v, do, 0.125, bias=-far)
    args = [t.cuda()[None, :, None] for t in (q, k, v)]
    slopes = torch.tensor([-1.0], device="cuda")
    o, lse = seq.attention(*args, slopes=slopes, return_lse=True)
    grads = seq.attention_backward(do.cuda()[None, :, None], *args, o, lse, slopes=slopes)
    _close("lse", lse[0, 0], *ref["lse"])
    for name, t in zip(("o", "dq", "dk", "dv"), (o,) + grads):
        _close(name, t[0, :, 0], *ref[name])


# ---- saturated scores -----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_gradient_of_saturated_scores(type, sign):
    """Every score is 6 to 9 times the cap before it is capped (16 bits: 7.5 to 9): what is left of the gradient is the cap's derivative,
    far below 1."""
    import torch
    from paper_2206_08720_amd import seq
    n, rows, cap, scale = 70, 40, 2.0, 0.125
    q, k = torch.zeros(rows, 64), _rand((n, 64), 980)
    q[:, 0] = 16.0 * sign
    k[:, 0] = torch.linspace(6.0 if type == "f32" else 7.5, 9.0, n)
    q, k, v, do = (t.to(_types()[type]) for t in (q, k, _rand((n, 64), 981), _rand((rows, 64), 982)))
    args = [t.cuda()[None, :, None] for t in (q, k, v)]
    o, lse = seq.attention(*args, softcap=cap, scale=scale, return_lse=True)
    grads = seq.attention_backward(do.cuda()[None, :, None], *args, o, lse, softcap=cap, scale=scale)
    ref = _one_head(type, q, k, v, do, scale, cap)
    for name, t in zip(("o", "dq", "dk", "dv"), (o,) + grads):
        _close(name, t[0, :, 0], *ref[name])


# ---- norms of rows whose squares leave fp32's range -----------------------------------------------------------------

@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(5, 96), (4, 785), (3, 2048), (2, 12289), (2, 32768)])
@pytest.mark.parametrize("size,eps", [(1e25, 1e-6), (5e37, 1e-6), (1e-30, 0.0), (3e-25, 1e-44)])
def test_rms_norm_of_any_size(type, rows, n, size, eps):
    """h of 1e25 has squares past fp32's largest, h of 1e-30 below its smallest; ordinary rows stand beside them.  The 8-bit
    form's y goes through the same numbers.  Tiny numbers: fp32's smallest step, 2^-149, in what is stored."""
    import torch
    from paper_2206_08720_amd import seq
    x, res, dy, dh = (_rand((rows, n), 990 + i, type) for i in range(4))
    x[0], res[0] = x[0].float().clamp(-3, 3) * size, res[0].float().clamp(-3, 3) * size
    dy, dh = dy * (1e3 if size > 1 else 1e-3), dh * (1 / size)
    w = (1 + 0.1 * _rand((n,), 995)).to(_types()[type])
    y, h = seq.rms_norm(x.cuda(), w.cuda(), residual=res.cuda(), eps=eps)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    ref = _norm_reference(x, res, w, eps, type, dy, dh, h.cpu())
    _close("y", y, *ref["y"])
    dx, dw = seq.rms_norm_backward(dy.cuda(), h, w.cuda(), dh=dh.cuda(), eps=eps)
    _close("dx", dx, ref["dx"][0], ref["dx"][1] + 2.0 ** -133)
    val, tol = ref["dw"]
    _close("dw", dw, val, tol)
    _, scale, _ = seq.rms_norm_e4m3(x.cuda(), w.cuda(), residual=res.cuda(), eps=eps)
    most = ref["y"][0].abs().max(1).values
    _close("scale", scale, most / 448, 2 * (n + 16) * E * most / 448)
