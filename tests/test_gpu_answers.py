"""The operators that a sequence model answers with, together and in the calls that a program makes of them: prompts and tokens over
a cache in pages, lengths of all kinds dealt out to the workgroups, streams, graphs, shared pages, refusals (paper_2206_08720_amd.seq).

The tolerances are those of tests/test_gpu_seq.py and tests/test_gpu_cache.py, or derived beside a test."""
import math

import pytest

from tests.test_gpu_cache import _attend, _empty, _fill, _ints, _sequence, _tables, _values
from tests.test_gpu_seq import U, _close, _oracle, _rand, _types

pytestmark = pytest.mark.gpu


# ---- a run of them ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("type,e4m3,page", [("bf16", False, 16), ("f32", False, 8), ("f16", True, 32), ("bf16", True, 64)])
def test_prompts_then_tokens(type, e4m3, page):
    """Prompts of lengths of their own in two parts, then tokens one by one: each step's attention against 64 bits over the cache as
    it stands, the cache against the turned keys, and the tokens' log probabilities against the logits that came out."""
    import torch
    from paper_2206_08720_amd import seq
    B, H, Hk, D, vocab = 3, 4, 2, 64, 517
    table = seq.rotary_table(200, D)
    most = (160 + page - 1) // page
    cache, pages = _empty(B * most, page, Hk, D, type, e4m3), _tables(B, most, B * most, 1)
    lens = torch.zeros(B, dtype=torch.int32)
    head = _rand((H * D, vocab), 3, "f32", 0.1).cuda()
    steps = [[37, 5, 64], [1, 30, 40]] + [[1, 1, 1]] * 3 + [[1, 0, 1]]
    stored = [[[] for _ in range(B)] for _ in range(2)]
    for s, new in enumerate(steps):
        n = max(new)
        q, k, v = _rand((B, n, H + 2 * Hk, D), 10 + s, type).split((H, Hk, Hk), 2)
        q1 = seq.cache_append(cache, pages.cuda(), lens.cuda(), k.cuda(), v.cuda(), q=q.cuda(), table=table, new_lens=_ints(new))
        at = lens[:, None] + torch.arange(n).int()
        want, want_k = seq.rotary(q.cuda(), table, at.cuda(), k=k.cuda())
        for b in range(B):
            if type == "f16":
                # a fused multiply-add may round to fp16 at once or by way of fp32: both are a rounding (u |y|) of a value within
                # 3 2^-24 (|u1 c| + |u2 s|) of the exact one, with magnitudes below 6
                ref = want[b, :new[b]].cpu().double()
                _close("q", q1[b, :new[b]], ref, 2 * U[type] * ref.abs() + 6 * 2.0 ** -24 * 12 + 2.0 ** -24)
            else:
                assert torch.equal(q1[b, :new[b]], want[b, :new[b]])          # the same turn as rotary's, to the last bit
            for i in range(new[b]):
                stored[0][b].append(want_k[b, i].cpu().double())
                stored[1][b].append(v[b, i].double())
        lens += _ints(new).cpu()
        o, lse = seq.attention_cached(q1, cache, pages.cuda(), lens.cuda(), q_lens=_ints(new), return_lse=True)
        kc, vc = _values(cache)
        for b in range(B):
            m, held = new[b], int(lens[b])
            kb, vb = _sequence(kc, pages, b, held, page), _sequence(vc, pages, b, held, page)
            for c, x in ((0, kb), (1, vb)):
                ref = torch.stack(stored[c][b])
                # 16 bits: the turned key as rotary rounds it.  8 bits: 2^-4, and 2^-10 of the page's scale (amax / 224 at most)
                tol = 2.0 ** -4 * (1 + U[type]) * ref.abs() + 2.0 ** -10 * ref.abs().max() / 224 * 2 + U[type] * ref.abs() if e4m3 else torch.zeros_like(ref)
                _close("kv"[c], x, ref, tol)
            if m:
                ref = _oracle(q1[b:b + 1, :m].cpu(), kb[None], vb[None], type, causal=True)
                _close("o", o[b:b + 1, :m], *ref["o"])
                _close("lse", lse[b:b + 1, :, :m], *ref["lse"])
        logits = (o[:, 0].flatten(1).float() @ head).to(_types()[type])
        tokens = torch.tensor([s, 100 + s, 500], dtype=torch.int32)
        got = seq.token_logprobs(logits, tokens.cuda(), top=4)
        ref = torch.log_softmax(logits.cpu().double(), 1)
        # 517 terms: (4 * 30 + 517 / 256 + 50 + 8) 2^-24 where |x - m| stays below 30
        _close("logp", got.logp, ref[torch.arange(B), tokens.long()], torch.full((B,), 200 * 2.0 ** -24).double())
        order = torch.sort(logits.cpu().float(), dim=1, descending=True, stable=True).indices[:, :4]
        assert torch.equal(got.top_tokens.cpu().long(), order)


def test_the_cache_gives_what_the_whole_sequence_gives():
    """One call of `attention` over dense keys and one over the same keys in pages; fp32, where both form the same products."""
    import torch
    from paper_2206_08720_amd import seq
    q, k, v = (_rand((2, 300, h, 64), 30 + h, "f32").cuda() for h in (4, 2, 2))
    cache, pages = seq.paged_cache(40, 16, 2, 64, torch.float32), _tables(2, 19, 40, 2).cuda()
    assert seq.cache_append(cache, pages, _ints([0, 0]), k, v) is None
    dense = seq.attention(q, k, v, causal=True)
    paged = seq.attention_cached(q, cache, pages, _ints([300, 300]))
    assert float((dense - paged).abs().max()) <= 2.0 ** -20 * float(v.abs().max())
    parts = torch.cat([seq.attention_cached(q[:, a:b].contiguous(), cache, pages, _ints([b, b])) for a, b in ((0, 1), (1, 40), (40, 300))], 1)
    assert float((parts - paged).abs().max()) <= 2.0 ** -20 * float(v.abs().max())


# ---- lengths that are dealt out ------------------------------------------------------------------------------------

UNEVEN = [
    # type, e4m3, H, Hk, D, page, capacity, k_lens, q_len, q_lens: one long sequence among short ones, empty ones, more sequences than threads,
    # row tiles of all lengths, queries that run past the keys, nearly as many sequences and heads as workgroups
    ("bf16", False, 8, 2, 128, 16, 6016, [6000, 1, 0, 33, 700, 32, 31, 2], 1, None, {}),
    ("bf16", True, 8, 2, 128, 64, 6016, [6000, 1, 0, 33, 700, 32, 31, 2], 1, None, {}),
    ("f16", True, 4, 4, 64, 16, 9600, [3, 9555, 0, 0, 9599], 2, [2, 1, 1, 0, 2], {}),
    ("f32", True, 4, 1, 128, 32, 2048, [2048, 5, 900], 3, None, {}),
    ("f32", False, 4, 1, 64, 32, 2048, [2048, 5, 900], 3, None, {"softcap": 9.0}),
    ("bf16", True, 4, 1, 128, 32, 1600, [1600, 300, 0, 77], 150, [150, 150, 3, 0], {}),
    ("bf16", False, 4, 1, 64, 8, 1600, [1600, 300, 0, 77], 150, [150, 150, 3, 100], {"causal": False}),
    ("f16", True, 2, 1, 80, 16, 1040, [1040, 200, 31], 300, [300, 200, 100], {"slopes": True}),
    ("f32", False, 2, 1, 64, 16, 800, [800, 100], 200, [133, 200], {}),
    ("bf16", True, 1, 1, 64, 128, 12800, [12800], 1, None, {}),
    ("bf16", False, 8, 8, 128, 16, 1024, [i * 397 % 1025 for i in range(31)], 1, None, {}),
    ("bf16", True, 8, 8, 128, 16, 2048, [i * 797 % 2049 for i in range(31)], 1, None, {}),
]


@pytest.mark.parametrize("case", UNEVEN, ids=lambda c: f"{c[0]}{'-e4m3' if c[1] else ''}-{c[8]}x{c[6]}-{c[2]}.{c[3]}.{c[4]}-{'.'.join(c[10])}")
def test_uneven_lengths(case):
    _attend(case, seed=700)


def test_many_sequences():
    """More sequences than a workgroup has threads, so that a thread counts several of them; and so many row tiles that each has a workgroup."""
    import torch
    from paper_2206_08720_amd import seq
    for B, Hk, capacity in ((700, 1, 1024), (1500, 4, 640)):
        g = torch.Generator().manual_seed(B)
        lens = [int(x) for x in torch.randint(0, capacity + 1, (B,), generator=g)]
        cache = _empty(64, 32, Hk, 64, "bf16", False)
        pages = torch.randint(0, 64, (B, capacity // 32), generator=g).int()       # pages that sequences share
        for t, seed in ((cache.k, 1), (cache.v, 2)):
            t.copy_(_rand(tuple(t.shape), 800 + seed, "bf16").cuda())
        q = _rand((B, 1, 2 * Hk, 64), 803, "bf16")
        o = seq.attention_cached(q.cuda(), cache, pages.cuda(), _ints(lens))
        k, v = _values(cache)
        for b in list(range(0, B, 97)) + [B - 1]:
            ref = _oracle(q[b:b + 1], _sequence(k, pages, b, lens[b], 32)[None], _sequence(v, pages, b, lens[b], 32)[None], "bf16")
            _close("o", o[b:b + 1], *ref["o"])
        assert torch.equal(o, seq.attention_cached(q.cuda(), cache, pages.cuda(), _ints(lens)))   # nothing depends on timing


# ---- streams, graphs, devices ----------------------------------------------------------------------------------------

def _step(seq, cache, pages, lens, x, table, tokens):
    k, v, q = x[:, :, :2], x[:, :, 2:4], x[:, :, 4:]
    q = seq.cache_append(cache, pages, lens, k, v, q=q, table=table)
    o, lse = seq.attention_cached(q, cache, pages, lens + x.shape[1], return_lse=True)
    logits = o.flatten(2).flatten(0, 1)
    got = seq.token_logprobs(logits, tokens, top=3)
    d = seq.token_logprobs_backward(got.logp, got.entropy, logits, tokens, got.lse, got.entropy)
    return (q, o, lse, *got, d)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n", [1, 40])
def test_graph_replays_match_eager(e4m3, n):
    """Two graphs of a step over one cache, replayed in turn, with eager calls between; lengths, keys and pages change under them."""
    import torch
    from paper_2206_08720_amd import seq
    B = 5
    make = lambda: seq.paged_cache(B * 130, 32, 2, 64, torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    cache, eager = make(), make()
    table, tokens = seq.rotary_table(4200, 64), _ints([7 * i % 500 for i in range(B * n)])
    pages, lens, x = _tables(B, 130, B * 130, 3).cuda(), _ints([0, 3000, 31, 500, 4000]), _rand((B, n, 12, 64), 40, "bf16").cuda()
    for c in (cache, eager):
        for t in (c.k, c.v):
            (t.view(torch.uint8) if e4m3 else t).copy_((_rand(tuple(t.shape), 41, "f32").cuda()).to(t.dtype).view(torch.uint8) if e4m3
                                                      else _rand(tuple(t.shape), 41, "bf16").cuda())
        if e4m3:
            c.k_scale.fill_(1.0)
            c.v_scale.fill_(0.5)
    run = lambda c: _step(seq, c, pages, lens, x, table, tokens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(cache)
    run(eager)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(cache))
        graphs.append(g)
    for r in range(6):
        x.copy_(_rand((B, n, 12, 64), 50 + r, "bf16", 1.0 + r))
        lens.copy_(_ints([r * n, 3000 + r, 31, 900 * (r % 2), 4000]))
        pages.copy_(_tables(B, 130, B * 130, 60 + r // 2).cuda())
        graphs[r % 2].replay()
        torch.cuda.synchronize()
        for a, b in zip(outs[r % 2], run(eager)):
            assert torch.equal(a, b)
        for a, b in zip(cache, eager):
            assert a is None or torch.equal(a.view(torch.uint8) if e4m3 else a, b.view(torch.uint8) if e4m3 else b)


def test_streams():
    """The calls run on the stream that they are given, and their tensors stay until it has passed them."""
    import torch
    from paper_2206_08720_amd import seq
    cache = seq.paged_cache(64, 16, 2, 64, torch.bfloat16)
    pages, lens, table = _tables(2, 32, 64, 4).cuda(), _ints([100, 0]), seq.rotary_table(600, 64)
    k, v, q = (_rand((2, 50, h, 64), 70 + h, "bf16").cuda() for h in (2, 2, 4))
    tokens = _ints([5, 6])
    q0 = seq.cache_append(cache, pages, lens, k, v, q=q, table=table)
    o0 = seq.attention_cached(q0, cache, pages, lens + 50)
    l0 = seq.token_logprobs(o0[:, -1].flatten(1), tokens, top=2)
    d0 = seq.token_logprobs_backward(l0.logp, None, o0[:, -1].flatten(1), tokens, l0.lse, l0.entropy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache2 = seq.PagedCache(torch.zeros_like(cache.k), torch.zeros_like(cache.v))
    side.wait_stream(torch.cuda.current_stream())
    q1 = seq.cache_append(cache2, pages, lens, k, v, q=q, table=table, stream=side)
    o1 = seq.attention_cached(q1, cache2, pages, _ints([150, 50]), stream=side)
    with torch.cuda.stream(side):
        row = o1[:, -1].flatten(1)
    l1 = seq.token_logprobs(row, tokens, top=2, stream=side)
    d1 = seq.token_logprobs_backward(l1.logp, None, row, tokens, l1.lse, l1.entropy, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(q0, q1) and torch.equal(o0[1], o1[1]) and torch.equal(l0.logp[1], l1.logp[1]) and torch.equal(d0[1], d1[1])


# ---- what is refused, and what counts as written -----------------------------------------------------------------------

def test_refusals():
    import torch
    from paper_2206_08720_amd import _lib, seq
    cache = seq.paged_cache(8, 16, 2, 64)
    e4m3 = seq.paged_cache(8, 16, 2, 64, torch.float8_e4m3fn)
    pages, lens = _tables(2, 3, 8, 1).cuda(), _ints([0, 0])
    k = torch.zeros(2, 5, 2, 64, device="cuda").bfloat16()
    q, logits, tokens = k, torch.zeros(4, 100, device="cuda"), _ints([1, 2, 3, 4])
    table = seq.rotary_table(50, 64)
    P = seq.PagedCache
    for call in (lambda: seq.paged_cache(8, 12, 2, 64), lambda: seq.paged_cache(8, 4, 2, 64), lambda: seq.paged_cache(0, 16, 2, 64),
                 lambda: seq.paged_cache(8, 16, 2, 64, torch.int8), lambda: seq.paged_cache(8, 16, 2, 64, device="cpu"),
                 lambda: seq.cache_append(cache, pages, lens.long(), k, k), lambda: seq.cache_append(cache, pages, None, k, k),
                 lambda: seq.cache_append(cache, pages[:1], lens, k, k), lambda: seq.cache_append(cache, pages[:, ::2], lens, k, k),
                 lambda: seq.cache_append(cache, pages, lens, k.float(), k.float()), lambda: seq.cache_append(cache, pages, lens, k, k[:, :4]),
                 lambda: seq.cache_append(cache, pages, lens, k[:, :, :1], k[:, :, :1]), lambda: seq.cache_append(cache, pages, lens, k[..., :32], k[..., :32]),
                 lambda: seq.cache_append(cache, pages, lens, k, k, positions=_ints([[0] * 5] * 2)), lambda: seq.cache_append(cache, pages, lens, k, k, q=q[..., :32]),
                 lambda: seq.cache_append(P(cache.k, cache.v, e4m3.k_scale, None), pages, lens, k, k), lambda: seq.cache_append(P(e4m3.k, e4m3.v), pages, lens, k, k),
                 lambda: seq.cache_append(P(e4m3.k, e4m3.v, e4m3.k_scale[:4], e4m3.v_scale), pages, lens, k, k),
                 lambda: seq.cache_append(P(e4m3.k, cache.v, e4m3.k_scale, e4m3.v_scale), pages, lens, k, k),
                 lambda: seq.cache_append(cache, pages, lens, k.cpu(), k), lambda: seq.cache_append(cache, pages, lens, k, k, table=table.double()),
                 lambda: seq.attention_cached(q, cache, pages, None), lambda: seq.attention_cached(q[..., :32], cache, pages, lens),
                 lambda: seq.attention_cached(q, cache, pages, lens, q_lens=lens[:1]), lambda: seq.attention_cached(q, cache, pages, lens, slopes=torch.zeros(3, device="cuda")),
                 lambda: seq.attention_cached(q, cache, pages.long(), lens), lambda: seq.attention_cached(q, cache, pages, lens, out=q[:1]),
                 lambda: seq.token_logprobs(logits, None), lambda: seq.token_logprobs(logits, tokens.long()), lambda: seq.token_logprobs(logits, tokens[:3]),
                 lambda: seq.token_logprobs(logits, tokens.cpu(), stream=torch.cuda.Stream()), lambda: seq.token_logprobs(logits, [1, 2, 3, 4], stream=torch.cuda.Stream()),
                 lambda: seq.token_logprobs_backward(tokens.cpu().float(), None, logits, tokens, torch.zeros(4, 2, device="cuda"), tokens.float(), stream=torch.cuda.Stream()),
                 lambda: seq.token_logprobs(logits, tokens, top=101), lambda: seq.token_logprobs(logits, tokens, top=-1), lambda: seq.token_logprobs(logits.double(), tokens),
                 lambda: seq.token_logprobs(logits.cpu(), tokens), lambda: seq.token_logprobs(logits[:, :0], tokens),
                 lambda: seq.token_logprobs_backward(tokens.float(), None, logits, tokens, torch.zeros(4, device="cuda"), tokens.float()),
                 lambda: seq.token_logprobs_backward(None, None, logits, tokens, None, tokens.float()),
                 lambda: seq.token_logprobs_backward(tokens.float(), None, logits[:1].expand(4, 100), tokens, torch.zeros(4, 2, device="cuda"), tokens.float(), inplace=True)):
        with pytest.raises((TypeError, ValueError)):
            call()
    for call in (lambda: seq.attention_cached(q[:, :, :1], cache, pages, lens), lambda: seq.attention_cached(q, cache, pages, lens, scale=-1.0),
                 lambda: seq.attention_cached(q, cache, pages, lens, out=q), lambda: seq.token_logprobs(logits, tokens, scale=0.0),
                 lambda: seq.cache_append(cache, pages, lens, cache.k[:2, :5], k), lambda: seq.cache_append(cache, pages, lens, k, k, table=seq.rotary_table(50, 66)),
                 lambda: seq.cache_append(P(cache.k[:1].expand(8, 16, 2, 64), cache.v), pages, lens, k, k),
                 lambda: seq.cache_append(P(cache.k, cache.k), pages, lens, k, k)):
        with pytest.raises(_lib.NTKError):
            call()
    # nothing to do: no tokens, no sequences, no places
    assert seq.cache_append(cache, pages, lens, k[:, :0], k[:, :0]) is None
    assert seq.attention_cached(q[:0], cache, pages[:0], lens[:0]).shape == (0, 5, 2, 64)
    o, lse = seq.attention_cached(q, cache, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), lens, return_lse=True)
    assert (o == 0).all() and (lse == -math.inf).all()
    seq.cache_append(cache, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), lens, k + 1, k + 1)
    assert (cache.k == 0).all() and (cache.v == 0).all()
    none = seq.token_logprobs(logits[:0], tokens[:0], top=3)
    assert none.logp.shape == (0,) and none.top_tokens.shape == (0, 3)


def test_gradients_are_not_lost_in_silence():
    """None of the calls is recorded: results of tensors that require a gradient say so, and what is written counts as changed."""
    import torch
    from paper_2206_08720_amd import seq
    cache = seq.paged_cache(8, 16, 2, 64, torch.float32)
    pages, lens, tokens = _tables(2, 3, 8, 1).cuda(), _ints([0, 0]), _ints([1, 2])
    k, p = torch.randn(2, 5, 2, 64, device="cuda"), torch.randn(2, 5, 2, 64, device="cuda", requires_grad=True)
    before = [t._version for t in cache[:2]]
    q = seq.cache_append(cache, pages, lens, k, k, q=p)
    assert all(t._version > b for t, b in zip(cache[:2], before))
    o = seq.attention_cached(p, cache, pages, lens + 5)
    logits = torch.randn(2, 50, device="cuda", requires_grad=True)
    got = seq.token_logprobs(logits, tokens, top=2)
    d = seq.token_logprobs_backward(tokens.float(), None, logits, tokens, got.lse.detach(), got.entropy.detach())
    for t in (q, o, got.logp, got.entropy, got.top_logp, d):
        with pytest.raises(RuntimeError, match="gradient"):
            t.sum().backward()
    assert p.grad is None and logits.grad is None
    for call in (lambda: seq.cache_append(cache, pages, lens, p, k), lambda: seq.attention_cached(k, cache, pages, lens, out=p),
                 lambda: seq.token_logprobs_backward(tokens.float(), None, logits, tokens, got.lse, got.entropy, inplace=True)):
        with pytest.raises(RuntimeError):
            call()
    with torch.no_grad():
        assert not seq.token_logprobs(logits, tokens).logp.requires_grad and seq.cache_append(cache, pages, lens, p, p) is None
