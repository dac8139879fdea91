"""The cache in pages and the attention over it (paper_2206_08720_amd.seq) against their definitions in 64 bits.

Tolerances, first order, with u the unit roundoff of the type and e = 2^-24:
* append in the arrays' type: a turned element is u1 c - u2 s in fp32 (two products and a sum, each rounded: at most 3 e (|u1 c| + |u2 s|)),
  then rounded once (u |y|, fp16 2^-25 more); a copied one is the same to the last bit;
* append in 8 bits: y / s is rounded to e4m3, 2^-4 |y| and half its smallest step, 2^-10 s.  Where a page's scale grows, its older
  cells lose half a smallest step of the new scale, 2^-10 s, and nothing else;
* attention: those of tests/test_gpu_seq.py over the values that the cache holds, which are given exactly.
"""
import math

import pytest

from tests.test_gpu_seq import E, TINY, U, _close, _oracle, _rand, _types

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _tables(B, most, pages, seed):
    """A table that deals out the cache's pages in no order."""
    import torch
    g = torch.Generator().manual_seed(seed)
    assert B * most <= pages
    return torch.randperm(pages, generator=g)[:B * most].view(B, most).int()


def _empty(pages, size, heads, dim, type, e4m3, layout="heads"):
    """A cache whose cells hold NaN (every one of 8 bits 0x7f): what no call wrote shows."""
    import torch
    from paper_2206_08720_amd import seq
    cells = torch.float8_e4m3fn if e4m3 else _types()[type]
    if layout == "heads":
        c = seq.paged_cache(pages, size, heads, dim, cells)
    else:                                   # [page, slot, head, dim] in memory; "odd": rows of an odd stride at an odd place
        pad = 3 if layout == "odd" else 0
        k, v = (torch.zeros(pages, size, heads, dim + pad, device="cuda", dtype=torch.uint8 if e4m3 else cells) for _ in range(2))
        if e4m3:
            k, v = k.view(cells), v.view(cells)
        if pad:
            k, v = k[..., 1:1 + dim], v[..., 1:1 + dim]
        s = [torch.full((pages, heads), math.nan, device="cuda") for _ in range(2)] if e4m3 else [None, None]
        c = seq.PagedCache(k, v, *s)
    for t in (c.k, c.v):
        if e4m3:
            t.view(torch.uint8).fill_(0x7f)
        else:
            t.fill_(math.nan)
    if e4m3:
        c.k_scale.fill_(math.nan)
        c.v_scale.fill_(math.nan)
    return c


def _values(cache):
    """(k, v) as they stand, in 64 bits on the CPU."""
    out = []
    for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = t.cpu().double()
        out.append(x if s is None else x * s.cpu().double()[:, None, :, None])
    return out


def _sequence(values, table, b, n, size):
    """Places 0 .. n - 1 of sequence b: [n, heads, dim]."""
    import torch
    at = torch.arange(n)
    return values[table[b].long()[at // size], at % size]


def _turn(x, pos, table, interleaved):
    """(x turned, |u1 c| + |u2 s|) in 64 bits; x [n, heads, dim], pos [n]."""
    import torch
    if table is None:
        return x.double(), torch.zeros(x.shape, dtype=torch.float64)
    rot = 2 * table.shape[1]
    t = torch.full((len(pos), rot // 2, 2), math.nan).double()
    there = (pos >= 0) & (pos < table.shape[0])
    t[there] = table.cpu().double()[pos[there].long()]
    c, s = t[:, None, :, 0], t[:, None, :, 1]
    i = torch.arange(rot // 2)
    iu, iv = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    y, mag = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    u, v = x.double()[..., iu], x.double()[..., iv]
    y[..., iu], y[..., iv] = u * c - v * s, v * c + u * s
    mag[..., iu], mag[..., iv] = (u * c).abs() + (v * s).abs(), (v * c).abs() + (u * s).abs()
    return y, mag


APPEND = [
    # type, e4m3, B, held, new, H, Hk, D, rot, page, options
    ("bf16", False, 1, [0], [1], 1, 1, 64, 64, 16, {}),
    ("bf16", False, 3, [5, 0, 37], [20, 1, 9], 4, 2, 128, 128, 16, {}),
    ("f16", False, 2, [0, 100], [33, 0], 2, 2, 80, 32, 32, {"interleaved": True}),
    ("f32", False, 2, [3, 4], [7, 2], 3, 1, 37, 36, 8, {}),
    ("f32", False, 2, [3, 9], [7, 2], 4, 1, 48, 48, 8, {"positions": True}),
    ("bf16", False, 2, [7, 15], [4, 4], 0, 2, 96, 0, 8, {}),
    ("bf16", False, 1, [2], [36], 2, 1, 128, 64, 8, {"layout": "slots"}),
    ("bf16", True, 1, [0], [1], 1, 1, 64, 64, 16, {}),
    ("bf16", True, 3, [5, 0, 37], [20, 1, 9], 4, 2, 128, 128, 16, {}),
    ("f16", True, 2, [0, 100], [33, 0], 2, 2, 80, 32, 32, {"interleaved": True}),
    ("f16", True, 2, [63, 1], [66, 70], 2, 3, 128, 128, 64, {"interleaved": True}),
    ("f32", True, 2, [3, 4], [7, 2], 3, 1, 37, 36, 8, {}),
    ("f32", True, 1, [0], [700], 1, 2, 64, 48, 512, {}),
    ("bf16", True, 2, [7, 15], [4, 4], 0, 2, 72, 16, 8, {"positions": True}),
    ("bf16", True, 1, [2], [36], 2, 1, 128, 0, 8, {"layout": "slots"}),
    ("bf16", True, 2, [9, 3], [40, 12], 2, 2, 64, 64, 16, {"layout": "odd"}),
    ("bf16", False, 2, [9, 3], [40, 12], 2, 2, 64, 64, 16, {"layout": "odd"}),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{c[0]}{'-e4m3' if c[1] else ''}-{c[5]}.{c[6]}.{c[7]}-rot{c[8]}-page{c[9]}-{'.'.join(c[10])}")
def test_append(case):
    """Two calls: the second one's tokens, larger ones, begin where the first one's end."""
    import torch
    from paper_2206_08720_amd import seq
    type, e4m3, B, held, new, H, Hk, D, rot, size, opt = case
    u, tiny = U[type], TINY[type]
    length = max(new) + 2
    most = (max(held) + 2 * length + size - 1) // size
    table = seq.rotary_table(max(held) + 2 * length + 60, rot) if rot else None
    cache = _empty(B * most + 3, size, Hk, D, type, e4m3, opt.get("layout", "heads"))
    pages = _tables(B, most, B * most + 3, 50)
    lens = list(held)
    known = [{}, {}]                        # (sequence, place) -> (value, tolerance) of k and of v
    for step in range(2):
        g = torch.Generator().manual_seed(60 + step)
        qkv = _rand((B, length, H + 2 * Hk, D), 70 + step, type, std=1.0 + 9.0 * step)
        q, k, v = qkv.split((H, Hk, Hk), 2)
        pos = (torch.randint(0, max(held) + 2 * length + 60, (B, length), generator=g).int() if "positions" in opt
               else torch.tensor(lens).int()[:, None] + torch.arange(length).int())
        dev = qkv.cuda()
        dq, dk, dv = dev.split((H, Hk, Hk), 2)
        before = _values(cache)
        bytes_before = [t.view(torch.uint8).cpu().clone() if e4m3 else t.cpu().clone() for t in (cache.k, cache.v)]
        scales = [s.cpu().double() if e4m3 else None for s in (cache.k_scale, cache.v_scale)]
        got = seq.cache_append(cache, pages.cuda(), _ints(lens), dk, dv, q=dq if H else None, table=table, new_lens=_ints(new),
                               positions=pos.cuda() if "positions" in opt else None, interleaved=opt.get("interleaved", False))
        torch.cuda.synchronize()
        assert (got is None) == (H == 0)
        if H:
            want, tol = torch.zeros(q.shape).double(), torch.zeros(q.shape).double()
            for b in range(B):
                n = new[b]
                y, mag = _turn(q[b, :n], pos[b, :n], table, opt.get("interleaved", False))
                want[b, :n], tol[b, :n] = y, u * y.abs() + 3 * E * mag + torch.where(mag > 0, tiny, 0.0)
            _close("q", got, want, tol)
        after = _values(cache)
        for c, x in enumerate((k, v)):
            changed = torch.zeros(bytes_before[c].shape[:2], dtype=torch.bool)      # page, slot
            for b in range(B):
                y, mag = _turn(x[b, :new[b]], pos[b, :new[b]], table if c == 0 else None, opt.get("interleaved", False))
                for e in range(lens[b] // size, (lens[b] + new[b] - 1) // size + 1 if new[b] else 0):
                    page = int(pages[b, e])
                    lo, hi = max(lens[b], e * size), min(lens[b] + new[b], (e + 1) * size)
                    part, m = y[lo - lens[b]:hi - lens[b]], mag[lo - lens[b]:hi - lens[b]]
                    older = range(e * size, lo)
                    changed[page, lo - e * size:hi - e * size] = True
                    if e4m3:
                        s = 2.0 ** torch.ceil(torch.log2(part.abs().amax((0, 2)) / 448))
                        if lo > e * size and not torch.isnan(scales[c][page]).any():
                            s = torch.maximum(s, scales[c][page])
                        if lo == e * size or not torch.isnan(scales[c][page]).any():
                            now = (cache.k_scale, cache.v_scale)[c][page].cpu().double()
                            assert torch.equal(now, s), (now, s)
                        now = (cache.k_scale, cache.v_scale)[c][page].cpu().double()
                        tol = 2.0 ** -4 * part.abs() + (2.0 ** -10 * now)[:, None] + 3 * E * m
                        for p in older:
                            changed[page, p - e * size] = True
                            if (b, p) in known[c]:
                                _close("older", after[c][page, p - e * size], before[c][page, p - e * size],
                                       torch.where(now > scales[c][page], 2.0 ** -10 * now, 0.0)[:, None])
                    else:
                        tol = torch.where(m > 0, u * part.abs() + 3 * E * m + tiny, 0.0)
                    _close("kv"[c], after[c][page, lo - e * size:hi - e * size], part, tol)
                    for p in range(lo, hi):
                        known[c][b, p] = True
            now = (cache.k, cache.v)[c]
            now = now.view(torch.uint8).cpu() if e4m3 else now.cpu()
            same = (now == bytes_before[c]) if e4m3 else (now.view(torch.uint8) == bytes_before[c].view(torch.uint8)).all(-1, keepdim=True)
            assert bool(same.all(-1).all(-1)[~changed].all()), "a slot without a token changed"
        lens = [a + n for a, n in zip(lens, new)]


def test_append_drops_what_has_no_place():
    """Page numbers outside the cache and places past the table: no slot changes but those of the tokens that have one."""
    import torch
    from paper_2206_08720_amd import seq
    for e4m3 in (False, True):
        cache = _empty(5, 8, 2, 64, "bf16", e4m3)
        raw = [t.view(torch.uint8) if e4m3 else t for t in (cache.k, cache.v)]
        before = [t.clone() for t in raw]
        pages = _ints([[-1, 3, 5, 2], [2 ** 31 - 1, -2 ** 31, 7, 0]])
        x = torch.ones(2, 40, 2, 64, device="cuda").bfloat16()
        q = seq.cache_append(cache, pages, _ints([0, 25]), x, x, q=x)
        assert torch.equal(q, x)
        one = torch.zeros(5, 8, dtype=torch.bool, device="cuda")
        one[3], one[2], one[0, 1:] = True, True, True
        for t, was, now in zip(raw, before, _values(cache)):
            if e4m3:
                assert torch.equal(t[~one], was[~one])
            else:
                assert torch.isnan(t[~one]).all()
            assert (now[one.cpu()] == 1).all()
        # lens below zero count as 0, past the table as its end; counts are clamped to what is there
        seq.cache_append(cache, pages, _ints([-7, 2 ** 31 - 1]), 2 * x, 2 * x, new_lens=_ints([2 ** 31 - 1, 99]))
        for now in _values(cache):
            assert (now[3] == 2).all() and (now[2] == 2).all() and (now[0, 1:] == 1).all()


def test_append_values_at_the_edge():
    """In 8 bits: zeros, values that are not finite, subnormals, and fp16's largest."""
    import torch
    from paper_2206_08720_amd import seq
    x = torch.zeros(1, 4, 1, 16)
    x[0, 0, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 3.0])
    cache = _empty(1, 8, 1, 16, "f32", True)
    seq.cache_append(cache, _ints([[0]]), _ints([0]), x.cuda(), torch.zeros_like(x).cuda())
    k, v = _values(cache)
    assert torch.isnan(k[0, 0, 0, :3]).all() and k[0, 0, 0, 3] == 3.0 and (k[0, 1:4] == 0).all() and (v[0, :4] == 0).all()
    assert float(cache.k_scale[0, 0]) == 2.0 ** -7 and float(cache.v_scale[0, 0]) == 2.0 ** -126
    # zeros leave no scale behind: what comes next has its own
    y = torch.full((1, 1, 1, 16), 1e-3)
    seq.cache_append(cache, _ints([[0]]), _ints([2]), y.cuda(), y.cuda())
    v = _values(cache)[1]
    assert ((v[0, 2] - 1e-3).abs() <= 2.0 ** -4 * 1e-3).all() and (v[0, :2] == 0).all()
    top = torch.tensor([65504.0, -65504.0, 61440.0, 63000.0] * 4).half().view(1, 1, 1, 16)
    cache = _empty(1, 8, 1, 16, "f16", True)
    seq.cache_append(cache, _ints([[0]]), _ints([0]), top.cuda(), top.cuda())
    assert (_values(cache)[0][0, 0, 0] == torch.tensor([61440.0, -61440.0, 61440.0, 61440.0] * 4)).all()
    for type in ("f32", "bf16"):            # 2^128 would be the next one up
        most = torch.finfo(_types()[type]).max
        top = torch.tensor([most, -most, 1.875 * 2.0 ** 127, 1.5 * 2.0 ** 127] * 4).to(_types()[type]).view(1, 1, 1, 16)
        cache = _empty(1, 8, 1, 16, type, True)
        seq.cache_append(cache, _ints([[0]]), _ints([0]), top.cuda(), top.cuda())
        want = torch.tensor([1.875, -1.875, 1.875, 1.5] * 4).double() * 2.0 ** 127
        assert (_values(cache)[0][0, 0, 0] == want).all() and (_values(cache)[1][0, 0, 0] == want).all()
    tiny = torch.full((1, 1, 1, 16), 2.0 ** -140)
    cache = _empty(1, 8, 1, 16, "f32", True)
    seq.cache_append(cache, _ints([[0]]), _ints([0]), tiny.cuda(), tiny.cuda())
    assert float(cache.k_scale[0, 0]) == 2.0 ** -126 and (_values(cache)[0][0, 0] == 0).all()


# ---- attention ------------------------------------------------------------------------------------------------------

def _fill(cache, pages, lens, type, seed, std=1.0):
    """Random keys and values in the first lens[b] places, by a plain rounding here."""
    import torch
    size, Hk, D = cache.k.shape[1:]
    e4m3 = cache.k_scale is not None
    for c, (t, s) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        raw = t.view(torch.uint8) if e4m3 else t
        for b, n in enumerate(lens):
            for e in range((n + size - 1) // size):
                m = min(size, n - e * size)
                x = _rand((m, Hk, D), seed + 1000 * c + 97 * b + e, "f32", std * (1.0 + 3.0 * (e % 3))).to(_types()[type])
                page = int(pages[b, e])
                if e4m3:
                    scale = 2.0 ** torch.ceil(torch.log2(x.double().abs().amax((0, 2)) / 448)).float()
                    s[page] = scale.cuda()
                    x = (x.float() / scale[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
                raw[page, :m] = x.cuda()


CACHED = [
    # type, e4m3, H, Hk, D, page, capacity, k_lens, q_len, q_lens, options
    ("bf16", False, 1, 1, 64, 16, 16, [1], 1, None, {}),
    ("bf16", False, 8, 8, 64, 16, 800, [777, 300, 16], 1, None, {}),
    ("f16", False, 8, 2, 128, 8, 1040, [1030, 1, 0], 1, None, {}),
    ("f32", False, 6, 3, 128, 32, 544, [33, 515], 1, [1, 1], {"slopes": True}),
    ("bf16", False, 32, 1, 128, 64, 640, [600, 31], 1, None, {"softcap": 20.0}),
    ("bf16", False, 12, 2, 80, 16, 608, [600, 3], 5, [5, 3], {"softcap": 20.0}),
    ("bf16", False, 4, 2, 128, 16, 208, [200, 130], 200, [200, 77], {}),
    ("bf16", False, 4, 2, 64, 128, 512, [300, 500], 70, None, {"causal": False}),
    ("f16", False, 3, 1, 72, 32, 352, [333], 333, None, {"softcap": 30.0, "slopes": True}),
    ("f32", False, 2, 1, 40, 8, 168, [161, 20], 161, [161, 0], {}),
    ("f32", False, 2, 2, 128, 64, 704, [700], 96, [90], {"softcap": 15.0}),
    ("bf16", False, 2, 1, 37, 8, 104, [100], 100, None, {}),
    ("bf16", False, 2, 1, 64, 8, 104, [100, 64], 40, None, {"layout": "odd"}),
    ("bf16", True, 1, 1, 64, 16, 16, [1], 1, None, {}),
    ("bf16", True, 8, 8, 64, 16, 800, [777, 300, 16], 1, None, {}),
    ("f16", True, 8, 2, 128, 8, 1040, [1030, 1, 0], 1, None, {}),
    ("f32", True, 6, 3, 128, 32, 544, [33, 515], 1, [1, 1], {"slopes": True}),
    ("f32", True, 6, 3, 64, 16, 544, [33, 515], 1, None, {}),
    ("bf16", True, 32, 1, 128, 64, 640, [600, 31], 1, None, {"softcap": 20.0}),
    ("bf16", True, 12, 2, 80, 16, 608, [600, 3], 5, [5, 3], {"softcap": 20.0}),
    ("bf16", True, 4, 2, 128, 16, 208, [200, 130], 200, [200, 77], {}),
    ("bf16", True, 4, 2, 64, 128, 512, [300, 500], 70, None, {"causal": False}),
    ("f16", True, 3, 1, 72, 32, 352, [333], 333, None, {"softcap": 30.0, "slopes": True}),
    ("f16", True, 2, 1, 96, 64, 384, [333], 333, [40], {}),
    ("f32", True, 2, 1, 40, 8, 168, [161, 20], 161, [161, 0], {}),
    ("f32", True, 2, 2, 64, 64, 704, [700], 96, [90], {"softcap": 15.0}),
    ("f32", True, 2, 2, 128, 64, 704, [700], 96, [90], {}),
    ("bf16", True, 2, 1, 64, 8, 104, [100, 64], 40, None, {"layout": "odd"}),
    ("bf16", True, 2, 2, 48, 8, 104, [100, 37], 1, None, {}),
    ("f16", True, 8, 2, 64, 8, 104, [100, 37], 30, [30, 29], {}),
    ("bf16", True, 2, 1, 128, 16, 64, [64, 5], 4, [9, 5], {"layout": "slots"}),
    ("bf16", True, 4, 1, 128, 16, 9008, [9000], 17, None, {}),
]


def _attend(case, seed=300, spoil=None):
    import torch
    from paper_2206_08720_amd import seq
    type, e4m3, H, Hk, D, size, capacity, lens, sq, q_lens, opt = case
    B, most = len(lens), capacity // size
    cache = _empty(B * most + 2, size, Hk, D, type, e4m3, opt.get("layout", "heads"))
    pages = _tables(B, most, B * most + 2, seed)
    _fill(cache, pages, lens, type, seed)
    for b, n in enumerate(lens):            # entries past the last page may hold anything
        pages[b, (n + size - 1) // size:] = torch.tensor([-1, 2 ** 31 - 1, 0, 10 ** 6]).repeat(most)[:most - (n + size - 1) // size]
    if spoil:
        spoil(cache, pages)
    q = _rand((B, sq, H, D), seed + 1, type)
    options = {"softcap": opt.get("softcap", 0.0), "causal": opt.get("causal", True),
               "slopes": torch.tensor([2.0 ** (-8 * (h + 1) / H) for h in range(H)]) if opt.get("slopes") else None}
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in options.items()}
    o, lse = seq.attention_cached(q.cuda(), cache, pages.cuda(), _ints(lens), q_lens=None if q_lens is None else _ints(q_lens), return_lse=True, **dev)
    torch.cuda.synchronize()
    k, v = _values(cache)
    for b, n in enumerate(lens):
        m = sq if q_lens is None else min(max(q_lens[b], 0), sq)
        assert (o[b, m:] == 0).all() and (lse[b, :, m:] == -math.inf).all()
        if m:
            ref = _oracle(q[b:b + 1, :m], _sequence(k, pages, b, n, size)[None], _sequence(v, pages, b, n, size)[None], type, k_lens=[n], **options)
            _close("o", o[b:b + 1, :m], *ref["o"])
            _close("lse", lse[b:b + 1, :, :m], *ref["lse"])
    return o


@pytest.mark.parametrize("case", CACHED, ids=lambda c: f"{c[0]}{'-e4m3' if c[1] else ''}-{c[8]}x{c[6]}-{c[2]}.{c[3]}.{c[4]}-page{c[5]}-{'.'.join(c[10])}")
def test_attention_cached(case):
    _attend(case)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("sq", [1, 40])
def test_pages_that_the_cache_lacks_read_as_nan(e4m3, sq):
    """The queries that see such a page give NaN, and no others."""
    import torch
    from paper_2206_08720_amd import seq
    cache = _empty(8, 16, 1, 64, "bf16", e4m3)
    pages = _tables(2, 4, 8, 5)
    _fill(cache, pages, [64, 64], "bf16", 6)
    q = _rand((2, sq, 1, 64), 7, "bf16").cuda()
    good = seq.attention_cached(q, cache, pages.cuda(), _ints([64, 64]))
    for bad in (-1, 8, 2 ** 31 - 1, -2 ** 31):
        broken = pages.clone()
        broken[1, 3] = bad
        o = seq.attention_cached(q, cache, broken.cuda(), _ints([64, 64]))
        hidden = max(0, sq - 16)            # queries in front of the last page
        assert torch.equal(o[0], good[0]) and torch.equal(o[1, :hidden], good[1, :hidden]) and torch.isnan(o[1, hidden:]).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_hidden_values_that_are_not_finite(e4m3):
    """Causal rows do not see a later place's infinities and NaN."""
    import torch
    from paper_2206_08720_amd import seq
    cache = _empty(10, 16, 2, 64, "bf16", e4m3)
    pages = _tables(1, 10, 10, 8)
    _fill(cache, pages, [160], "bf16", 9)
    q = _rand((1, 160, 4, 64), 10, "bf16").cuda()
    good = seq.attention_cached(q, cache, pages.cuda(), _ints([160]))
    page, slot = int(pages[0, 100 // 16]), 100 % 16
    for t in (cache.k, cache.v):
        t = t.view(torch.uint8) if e4m3 else t
        t[page, slot, 1] = 0x7f if e4m3 else math.inf
    o = seq.attention_cached(q, cache, pages.cuda(), _ints([160]))
    assert torch.equal(o[:, :, :2], good[:, :, :2])                   # the other head
    assert torch.isfinite(o[0, :100].float()).all() and torch.equal(o[0, :100], good[0, :100])
    assert not torch.isfinite(o[0, 100:, 2:].float()).all(-1).any()


@pytest.mark.parametrize("sq", [1, 40])
def test_an_infinite_value_passes_the_join(sq):
    """A sequence cut into parts for many workgroups: +inf among the values of one channel is +inf there, and nothing elsewhere."""
    import torch
    from paper_2206_08720_amd import seq
    n, size = 9000, 16
    cache = _empty(570, size, 1, 64, "bf16", False)
    pages = _tables(1, 570, 570, 11)
    _fill(cache, pages, [n], "bf16", 12)
    q = _rand((1, sq, 4, 64), 13, "bf16")
    k, v = (_sequence(x, pages, 0, n, size)[None] for x in _values(cache))
    want, tol = _oracle(q, k, v, "bf16", causal=True)["o"]
    others = [d for d in range(64) if d != 1]
    for at in (0, 4500, n - sq):            # in the first part, in between, in the last one
        page, slot = int(pages[0, at // size]), at % size
        kept = cache.v[page, slot, 0, 1].clone()
        cache.v[page, slot, 0, 1] = math.inf
        o = seq.attention_cached(q.cuda(), cache, pages.cuda(), _ints([n]))
        cache.v[page, slot, 0, 1] = kept
        assert (o[..., 1] == math.inf).all()
        _close("o", o[..., others], want[..., others], tol[..., others])


def test_large_offsets():
    """A cache of 6 GiB: pages past 2^32 bytes, and strides past 2^31 elements."""
    import torch
    from paper_2206_08720_amd import seq
    for e4m3 in (False, True):
        pages, size, Hk, D = (1 << 18) + 9, 16, 4, 128
        kind = torch.uint8 if e4m3 else torch.bfloat16
        k = torch.empty(pages, Hk, size, D, dtype=kind, device="cuda").transpose(1, 2)
        k = k.view(torch.float8_e4m3fn) if e4m3 else k
        scales = [torch.ones(pages, Hk, device="cuda") for _ in range(2)] if e4m3 else [None, None]
        v = torch.empty_like(k.view(kind)).view(k.dtype)
        cache = seq.PagedCache(k, v, *scales)
        table = torch.tensor([[pages - 1, 3, pages - 2], [0, pages - 5, 7]]).int()
        x = _rand((2, 40, 2 * Hk, D), 20, "bf16")
        kk, vv = x.cuda().split((Hk, Hk), 2)
        seq.cache_append(cache, table.cuda(), _ints([0, 0]), kk, vv)
        q = _rand((2, 40, 8, D), 21, "bf16")
        o = seq.attention_cached(q.cuda(), cache, table.cuda(), _ints([40, 40]))
        one = seq.attention_cached(q[:, -1:].cuda(), cache, table.cuda(), _ints([40, 40]))
        for b in range(2):
            got = []
            for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
                y = torch.stack([t[int(table[b, p // size]), p % size].cpu().double() * (1 if s is None else s[int(table[b, p // size])].cpu().double()[:, None])
                                 for p in range(40)])
                got.append(y)
            assert float((got[0] - x[b, :, :Hk].double()).abs().max()) <= (2.0 ** -4 * 5.5 if e4m3 else 0.0)
            ref = _oracle(q[b:b + 1], got[0][None], got[1][None], "bf16", causal=True)
            _close("o", o[b:b + 1], *ref["o"])
            _close("one", one[b:b + 1], ref["o"][0][:, -1:], ref["o"][1][:, -1:])
        del k, v, cache
        torch.cuda.empty_cache()
