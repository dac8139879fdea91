"""Log probabilities of given tokens, entropy, alternatives and the gradient (paper_2206_08720_amd.seq) against their definitions in
64 bits.

Tolerances, first order, e = 2^-24, n = vocab, X = the largest scale |x|:
* x - m is formed from exact values with one rounding, times c = scale log2(e) (3 roundings of it), so 2^((x - m) c) is off by at most the
  relative 4 e |x - m| scale + 2 e; where |x - m| scale is over 150 the term is 0.  With the sums' roundings (a thread adds at most
  n / 256 + 32 terms in a row, the rest is a tree), l is off by the relative k = (4 * 150 + n / 256 + 50) e at the very worst, and
  by r = 4 e mean|x - m| scale + (n / 256 + 50) e when weighted by the terms, which is what is used;
* logp: (x_t - m) scale - log l: 3 e |(x_t - m) scale| + r + 2 e |log l| + e |logp|;
* lse: m as it is, log l off by r + 2 e |log l|;  entropy: log l - s / l: 3 r (1 + H + log l);
* dlogits: p off by the relative 4 e |x - m| scale + r + 3 e log l + 8 e; then u |d| of the type (fp16 2^-25 more).
"""
import math

import pytest

from tests.test_gpu_seq import E, TINY, U, _close, _rand, _types

pytestmark = pytest.mark.gpu


def _reference(logits, tokens, scale, type, top=0, dlogp=None, dentropy=None):
    """{name: (value, tolerance)}; rows in which everything is ruled out by their own rule."""
    import torch
    u, tiny = U[type], TINY[type]
    raw = logits.double()
    x, n = raw * scale, logits.shape[-1]
    rows = torch.arange(len(raw))
    none = (raw == -math.inf).all(1)
    m = torch.where(none, 0.0, x.max(1).values)
    d = torch.where(x == -math.inf, 0.0, x - m[:, None])
    ex = torch.where(x == -math.inf, 0.0, torch.exp(d))
    l = torch.where(none, 1.0, ex.sum(1))
    p = ex / l[:, None]
    H = l.log() - (p * d).sum(1)
    r = 4 * E * (p * d.abs()).sum(1) + (n / 256 + 50) * E
    t = tokens.long().clamp(0, n - 1)
    dt = torch.where(x[rows, t] == -math.inf, -math.inf, d[rows, t])
    logp = torch.where(none, -math.inf, dt - l.log())
    logp = torch.where(tokens < 0, 0.0, torch.where(tokens >= n, math.nan, logp))

    def about(v, dd):
        return torch.where(v == -math.inf, 0.0, 3 * E * dd.abs().nan_to_num(posinf=0.0) + r.view(-1, *[1] * (v.dim() - 1)) + 2 * E * l.log().abs().view(-1, *[1] * (v.dim() - 1)) + E * v.abs())

    out = {"logp": (logp, about(logp, dt)), "entropy": (torch.where(none, 0.0, H), 3 * r * (1 + H + l.log())),
           "lse": (torch.stack((raw.max(1).values, l.log()), 1), torch.stack((torch.zeros_like(r), r + 2 * E * l.log()), 1))}
    if top:
        which = torch.sort(raw + 0.0, dim=1, descending=True, stable=True).indices[:, :top]
        dd = torch.where(x.gather(1, which) == -math.inf, -math.inf, d.gather(1, which))
        lp = torch.where(none[:, None], -math.inf, dd - l.log()[:, None])
        out["top_logp"], out["top_tokens"] = (lp, about(lp, dd)), which.int()
    if dlogp is not None or dentropy is not None:
        gl = torch.zeros(len(raw)).double() if dlogp is None else torch.where(tokens < 0, 0.0, dlogp.double())
        gl = torch.where(tokens >= n, math.nan, gl)
        ge = torch.zeros(len(raw)).double() if dentropy is None else dentropy.double()
        hot = torch.zeros(x.shape).double()
        hot[rows[tokens >= 0], t[tokens >= 0]] = 1.0
        lp = torch.where(p > 0, d - l.log()[:, None], 0.0)
        a = gl[:, None] * (hot - p) - ge[:, None] * p * (lp + H[:, None])
        a = scale * torch.where(none[:, None] & ~(tokens >= n)[:, None], 0.0, a)
        rel = 4 * E * d.abs() + (r + 3 * E * l.log() + 8 * E)[:, None]
        mag = scale * p * (gl.abs()[:, None] + ge.abs()[:, None] * (1 + lp.abs() + H[:, None]))
        out["dlogits"] = (a, u * a.abs() + 4 * E * scale * gl.abs()[:, None] * hot + 2 * rel * mag.nan_to_num() + tiny + 2.0 ** -126)
    return out


def _run(logits, tokens, scale, type, top=0, gradient=True, seed=5, place=lambda t: t.cuda()):
    import torch
    from paper_2206_08720_amd import seq
    rows = len(logits)
    dlogp, dentropy = (_rand((rows,), seed + i) for i in range(2)) if gradient else (None, None)
    ref = _reference(logits, tokens, scale, type, top, dlogp, dentropy)
    x = place(logits)
    got = seq.token_logprobs(x, tokens.cuda(), top=top, scale=scale)
    have = {"logp": got.logp, "entropy": got.entropy, "lse": got.lse}
    if top:
        have["top_logp"] = got.top_logp
    if gradient:
        have["dlogits"] = seq.token_logprobs_backward(dlogp.cuda(), dentropy.cuda(), x, tokens.cuda(), got.lse, got.entropy, scale=scale)
    torch.cuda.synchronize()
    for name, t in have.items():
        _close(name, t, *ref[name])
    if top:
        assert got.top_tokens.dtype == torch.int32 and torch.equal(got.top_tokens.cpu(), ref["top_tokens"])
    else:
        assert got.top_logp is None and got.top_tokens is None
    return got


SIZES = [
    # type, rows, vocab, top, scale
    ("f32", 1, 1, 1, 1.0), ("f32", 3, 2, 2, 0.5), ("bf16", 5, 7, 3, 1.0), ("f16", 2, 64, 64, 2.0), ("bf16", 4, 1000, 5, 1.0),
    ("f32", 2, 1025, 1, 1.3), ("f16", 7, 5001, 20, 1.0), ("bf16", 1, 50001, 20, 1.4), ("f32", 3, 40003, 64, 1.0), ("bf16", 2, 131072, 20, 0.7),
    ("bf16", 300, 2049, 0, 1.0), ("f32", 33, 32768, 0, 1.0), ("f16", 1, 100000, 0, 1.0), ("bf16", 2000, 333, 4, 1.0),
]


@pytest.mark.parametrize("type,rows,vocab,top,scale", SIZES)
def test_logprobs(type, rows, vocab, top, scale):
    import torch
    logits = _rand((rows, vocab), 400, type, 3.0)
    tokens = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(1)).int()
    _run(logits, tokens, scale, type, top)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
def test_strides_and_places(type):
    """Rows of an odd stride at an odd place, leading dimensions, and a broadcast row."""
    import torch
    from paper_2206_08720_amd import seq
    logits, tokens = _rand((6, 3001), 410, type, 3.0), torch.arange(6).int() * 500

    def odd(t):
        w = torch.full((6, 3014), math.nan, dtype=t.dtype, device="cuda")
        w[:, 5:3006] = t
        return w[:, 5:3006]

    _run(logits, tokens, 1.0, type, 7, place=odd)
    # a row's sums are taken by 16 aligned bytes, so in another order where it starts elsewhere: each stands for itself
    ref = _reference(logits, tokens, 1.0, type, 7)

    def same(got, rows, lead):
        for name in ("logp", "entropy", "lse", "top_logp"):
            t = getattr(got, name)
            assert t.shape[:len(lead)] == lead
            _close(name, t.reshape(len(rows), *t.shape[len(lead):]), *(x[rows] for x in ref[name]))
        assert got.top_tokens.shape == (*lead, 7) and torch.equal(got.top_tokens.cpu().view(len(rows), 7), ref["top_tokens"][rows])

    same(seq.token_logprobs(logits.cuda().view(2, 3, 3001), tokens.cuda().view(2, 3), top=7), list(range(6)), (2, 3))
    same(seq.token_logprobs(logits[4].cuda(), tokens[4].cuda(), top=7), [4], ())
    same(seq.token_logprobs(logits[2:3].cuda().expand(6, 3001), tokens[2:3].cuda().expand(6), top=7), [2] * 6, (6,))


def test_rows_of_nothing_and_padding():
    """Everything ruled out; one token left; the type's lowest value; tokens that are padding or past the vocabulary."""
    import torch
    for type in ("f32", "bf16"):
        logits = _rand((9, 700), 420, type, 3.0)
        logits[0] = -math.inf
        logits[1] = -math.inf
        logits[1, 333] = 2.0
        logits[2] = torch.finfo(logits.dtype).min
        logits[3, 5:] = torch.finfo(logits.dtype).min
        logits[4, ::2] = -math.inf
        tokens = torch.tensor([3, 333, 10, 2, 4, -1, 700, -2 ** 31, 2 ** 31 - 1]).int()
        got = _run(logits, tokens, 1.0, type, 9)
        assert got.top_tokens[0].tolist() == list(range(9)) and got.top_tokens[1].tolist() == [333, 0, 1, 2, 3, 4, 5, 6, 7]
        _run(logits, tokens, 1.0, type, 0)


def test_not_finite():
    """A NaN or +inf makes its row's numbers NaN, not its neighbours'; NaN comes before all alternatives."""
    import torch
    from paper_2206_08720_amd import seq
    logits = _rand((3, 5000), 430, "f32", 3.0)
    good = seq.token_logprobs(logits.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda"), top=3)
    logits[1, 4321] = math.nan
    logits[1, 77] = math.inf
    got = seq.token_logprobs(logits.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda"), top=3)
    assert torch.isnan(got.logp[1]) and torch.isnan(got.entropy[1]) and torch.isnan(got.top_logp[1]).all() and got.top_tokens[1, :2].tolist() == [4321, 77]
    for a, b in zip(got, good):
        assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])
    d = seq.token_logprobs_backward(good.logp, None, logits.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda"), got.lse, got.entropy)
    assert torch.isnan(d[1]).all() and torch.isfinite(d[0]).all() and torch.isfinite(d[2]).all()


def test_ties_go_to_the_lowest_token():
    import torch
    from paper_2206_08720_amd import seq
    for n in (70, 5000, 131072):
        x = torch.zeros(2, n).bfloat16()
        x[1, ::2] = -0.0
        x[1, n - 3] = 1.0
        got = seq.token_logprobs(x.cuda(), torch.zeros(2, dtype=torch.int32, device="cuda"), top=64)
        assert got.top_tokens[0].tolist() == list(range(64)) and got.top_tokens[1].tolist() == [n - 3] + list(range(63))
    # logits that grow and fall along the row: every one is an alternative when it is met
    x = torch.arange(20000).float()
    for y in (x, -x):
        got = seq.token_logprobs(y.cuda()[None] / 100, torch.zeros(1, dtype=torch.int32, device="cuda"), top=64)
        assert got.top_tokens[0].tolist() == torch.sort(y, descending=True).indices[:64].tolist()


def test_large_logits_keep_their_differences():
    """Logits near 2^14 that differ by a few units: nothing large enters the sums."""
    import torch
    logits = (_rand((4, 3000), 440, "f32", 2.0) * 64).round() / 64 + 16384
    _run(logits, torch.arange(4).int(), 1.0, "f32", 5)


def test_gradient_against_differences():
    """Central differences in 64 bits of the formula's values; the operator's gradient is that of the formula."""
    import torch
    from paper_2206_08720_amd import seq
    x = _rand((2, 50), 450, "f32", 2.0)
    tokens, a, b, scale = torch.tensor([7, 31]).int(), _rand((2,), 451), _rand((2,), 452), 1.25

    def value(x):
        lp = torch.log_softmax(x * scale, 1)
        return (a.double() * lp[torch.arange(2), tokens.long()]).sum() - (b.double() * (lp.exp() * lp).sum(1)).sum()

    got = seq.token_logprobs(x.cuda(), tokens.cuda(), scale=scale)
    d = seq.token_logprobs_backward(a.cuda(), b.cuda(), x.cuda(), tokens.cuda(), got.lse, got.entropy, scale=scale).cpu().double()
    h = 2.0 ** -14
    for r in range(2):
        for j in range(0, 50, 7):
            p = x.double()
            p[r, j] += h
            q = x.double()
            q[r, j] -= h
            # the third derivative is below 4 scale^3 (|a| + 4 |b|); 64-bit values cancel to 2^-52 30 / h
            assert abs(float((value(p) - value(q)) / (2 * h)) - float(d[r, j])) <= 4 * 2 * 16 * h * h + 2.0 ** -52 * 60 / h + 2.0 ** -18
    only = seq.token_logprobs_backward(a.cuda(), None, x.cuda(), tokens.cuda(), got.lse, got.entropy, scale=scale)
    rest = seq.token_logprobs_backward(None, b.cuda(), x.cuda(), tokens.cuda(), got.lse, got.entropy, scale=scale)
    assert float(((only + rest).cpu().double() - d).abs().max()) <= 2.0 ** -20
    y = x.cuda()
    assert seq.token_logprobs_backward(a.cuda(), b.cuda(), y, tokens.cuda(), got.lse, got.entropy, scale=scale, inplace=True) is y
    assert torch.equal(y.cpu().double(), d)
