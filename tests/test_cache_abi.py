"""CPU-side checks of the paged cache's and the token probabilities' entry points (include/ntk_seq.h): bad arguments are refused on the
host, before any device call."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2206_08720_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2206_08720_amd.build import build
        build()
    return _lib.load()


P = 4096


def _view(place=1, b=1 << 20, n=256, h=64):
    from paper_2206_08720_amd import _lib
    return _lib.ntk_view(P * place, b, n, h)


def _cache(**kw):
    from paper_2206_08720_amd import _lib
    d = dict(dtype=_lib.NTK_BF16, pages=10, page_size=16, kv_heads=2, head_dim=64, k=_view(50, 4096, 128, 64), v=_view(60, 4096, 128, 64),
             k_scale=P * 70, v_scale=P * 71, page_table=P * 80, max_pages=4)
    d.update(kw)
    return _lib.ntk_cache(**d)


BAD_CACHES = [
    ({"dtype": 0}, "NTK_E_ARG"), ({"dtype": 4}, "NTK_E_ARG"), ({"dtype": -1}, "NTK_E_ARG"), ({"pages": -1}, "NTK_E_ARG"), ({"max_pages": -1}, "NTK_E_ARG"),
    ({"page_size": 0}, "NTK_E_UNSUPPORTED"), ({"page_size": 4}, "NTK_E_UNSUPPORTED"), ({"page_size": 24}, "NTK_E_UNSUPPORTED"),
    ({"page_size": 2048}, "NTK_E_UNSUPPORTED"), ({"kv_heads": 0}, "NTK_E_SHAPE"), ({"head_dim": 0}, "NTK_E_ARG"), ({"head_dim": 129}, "NTK_E_UNSUPPORTED"),
    ({"page_table": None}, "NTK_E_ARG"), ({"page_table": P + 2}, "NTK_E_ARG"), ({"max_pages": 1 << 27}, "NTK_E_UNSUPPORTED"),
    ({"k": "null"}, "NTK_E_ARG"), ({"v": "odd"}, "NTK_E_ARG"), ({"k": "negative"}, "NTK_E_ARG"),
    ({"dtype": 3, "k_scale": None}, "NTK_E_ARG"), ({"dtype": 3, "v_scale": P + 1}, "NTK_E_ARG"), ({"dtype": 3, "v_scale": P * 70}, "NTK_E_ARG")]


def _bad(change):
    from paper_2206_08720_amd import _lib
    views = {"null": _lib.ntk_view(0, 4096, 128, 64), "odd": _lib.ntk_view(P * 60 + 1, 4096, 128, 64), "negative": _lib.ntk_view(P * 50, 4096, -128, 64)}
    return {k: views.get(v, v) if isinstance(v, str) else v for k, v in change.items()}


def _append(lib, cache, dtype=1, b=2, n=3, h=4, lens=P * 2, news=None, k=1, v=1, q=1, qo=1, table=P * 3, max_pos=100, rot=64, positions=None):
    ref = lambda x, d: None if x is None else ctypes.byref(d if x == 1 else x)
    return lib.ntk_cache_append(dtype, b, n, h, None if cache is None else ctypes.byref(cache), lens, news, ref(k, _view(10)), ref(v, _view(20)), ref(q, _view(30)),
                                ref(qo, _view(40)), table, max_pos, rot, 0, positions, None)


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_cache_refusals(lib, change, code):
    from paper_2206_08720_amd import _lib
    bad = _cache(**_bad(change))
    assert _append(lib, bad) == getattr(_lib, code)
    assert "cache_append" in _lib.last_error()
    d = _lib.ntk_attention_desc(_lib.NTK_BF16, 2, 1, bad.max_pages * bad.page_size & 0x7fffffff, 4, bad.kv_heads, bad.head_dim, 1, 0.125, 0.0, P)
    v = ctypes.byref(_view(90))
    assert lib.ntk_attention_cached(ctypes.byref(d), ctypes.byref(bad), None, v, ctypes.byref(_view(91)), None, P, 1 << 40, None) < 0
    assert "attention" in _lib.last_error()


def test_append_refusals(lib):
    from paper_2206_08720_amd import _lib
    good = _cache()
    for bad in ({"dtype": 3}, {"b": -1}, {"n": -1}, {"h": -1}, {"lens": None}, {"lens": P + 1}, {"news": P + 2}, {"positions": P + 3}, {"k": None}, {"v": None},
                {"qo": None}, {"table": None}, {"table": P + 2}, {"max_pos": 0}, {"k": _view(10, n=-1)}, {"v": _lib.ntk_view(P * 20 + 1, 0, 0, 0)},
                {"qo": _view(30)}, {"qo": _view(10)}, {"qo": _view(40, h=63)}, {"qo": _view(40, b=0)}, {"qo": _view(50)}, {"k": _view(50)}, {"v": _view(60)}):
        assert _append(lib, good, **bad) == _lib.NTK_E_ARG, bad
    for rot in (-2, 63, 66):
        assert _append(lib, good, rot=rot) == _lib.NTK_E_SHAPE
    for cells in (_view(50, 4096, 128, 63), _view(50, 0, 128, 64), _view(50, 4096, 0, 64), _view(60, 4096, 128, 64)):
        assert _append(lib, _cache(k=cells)) == _lib.NTK_E_ARG
    assert _append(lib, None) == _lib.NTK_E_ARG
    assert _append(lib, good, b=1 << 16, n=1 << 16) == _lib.NTK_E_UNSUPPORTED
    assert _append(lib, good, h=1 << 30) == _lib.NTK_E_UNSUPPORTED
    assert _append(lib, _cache(max_pages=(1 << 26) - 200, page_size=32), b=1, n=10000) == _lib.NTK_E_UNSUPPORTED
    # nothing to do
    assert _append(lib, good, n=0) == _lib.NTK_OK and _append(lib, good, b=0, lens=None, k=None) == _lib.NTK_OK


def test_attention_cached_refusals(lib):
    from paper_2206_08720_amd import _lib
    c = _cache()

    def desc(**kw):
        d = dict(dtype=_lib.NTK_BF16, batch=2, q_len=1, k_len=64, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, softcap=0.0, k_lens=P)
        d.update(kw)
        return ctypes.byref(_lib.ntk_attention_desc(**d))

    def call(d, cache=c, q_lens=None, q=_view(90), o=_view(91), lse=None, work=P, size=1 << 40):
        ref = lambda x: None if x is None else ctypes.byref(x)
        return lib.ntk_attention_cached(d, ref(cache), q_lens, ref(q), ref(o), lse, work, size, None)

    for bad in ({"dtype": 3}, {"batch": -1}, {"scale": 0.0}, {"softcap": -1.0}, {"prefix": P}, {"docs": P}, {"k_lens": None}, {"k_lens": P + 2}, {"slopes": P + 2},
                {"dtype": 0}):
        assert call(desc(**bad)) == _lib.NTK_E_ARG, bad
    for bad in ({"kv_heads": 1}, {"heads": 3}, {"head_dim": 32}, {"k_len": 63}, {"k_len": 128}):
        assert call(desc(**bad)) == _lib.NTK_E_SHAPE, bad
    for bad in ({"cache": None}, {"q": None}, {"o": None}, {"o": _view(90)}, {"o": _view(50)}, {"o": _view(60)}, {"o": _view(91, h=63)}, {"q": _lib.ntk_view(P + 1, 0, 0, 0)},
                {"q_lens": P + 1}, {"lse": P + 1}):
        assert call(desc(), **bad) == _lib.NTK_E_ARG, bad
    assert lib.ntk_attention_cached_workspace(desc(), 2) == _lib.NTK_E_ARG
    assert lib.ntk_attention_cached_workspace(desc(head_dim=129), 1) == _lib.NTK_E_UNSUPPORTED
    assert lib.ntk_attention_cached_workspace(desc(q_len=1 << 28, heads=8), 1) == _lib.NTK_E_UNSUPPORTED
    assert lib.ntk_attention_cached_workspace(desc(q_len=0), 1) == 0 and lib.ntk_attention_cached_workspace(desc(batch=0), 3) == 0
    # ranges of a long cache need a workspace
    big, long = desc(k_len=65536), _cache(max_pages=4096)
    need = lib.ntk_attention_cached_workspace(big, 1)
    assert need > 0
    for work, size in ((None, need), (P, need - 1), (P + 4, need)):
        assert call(big, cache=long, work=work, size=size) == _lib.NTK_E_ARG
        assert "workspace" in _lib.last_error()
    # a large batch over large caches fits a launch
    assert lib.ntk_attention_cached_workspace(desc(batch=2048, k_len=1 << 20, heads=32, kv_heads=8, head_dim=128), 3) >= 0


def test_logprobs_refusals(lib):
    from paper_2206_08720_amd import _lib

    def call(dtype=1, rows=4, vocab=100, x=P, stride=100, t=P, scale=1.0, top=3, logp=P, entropy=P, lse=P, tl=P, tt=P, work=P, size=1 << 30):
        return lib.ntk_logprobs(dtype, rows, vocab, x, stride, t, scale, top, logp, entropy, lse, tl, tt, work, size, None)

    for bad in ({"dtype": 3}, {"rows": -1}, {"vocab": 0}, {"x": None}, {"t": None}, {"logp": None}, {"tl": None}, {"tt": None}, {"stride": 99}, {"top": -1}, {"top": 101},
                {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"scale": 3e38}, {"x": P + 1}, {"t": P + 2}, {"logp": P + 1},
                {"entropy": P + 1}, {"lse": P + 2}, {"tl": P + 2}, {"tt": P + 1}):
        assert call(**bad) == _lib.NTK_E_ARG, bad
    assert call(top=65) == _lib.NTK_E_UNSUPPORTED
    assert call(vocab=1 << 30, stride=1 << 30) == _lib.NTK_E_UNSUPPORTED and call(rows=1 << 40) == _lib.NTK_E_UNSUPPORTED
    assert call(rows=0, x=None) == _lib.NTK_OK
    need = lib.ntk_logprobs_workspace(1, 1, 131072, 5)
    assert need > 0 and lib.ntk_logprobs_workspace(1, 5000, 131072, 5) == 0
    for work, size in ((None, need), (P, need - 1), (P + 8, need)):
        assert call(rows=1, vocab=131072, stride=131072, top=5, work=work, size=size) == _lib.NTK_E_ARG

    def back(dtype=1, rows=4, vocab=100, x=P, stride=100, t=P, scale=1.0, lse=P, entropy=P, dl=P, de=P, out=2 * P, ostride=100):
        return lib.ntk_logprobs_bwd(dtype, rows, vocab, x, stride, t, scale, lse, entropy, dl, de, out, ostride, None)

    for bad in ({"dtype": -1}, {"x": None}, {"t": None}, {"lse": None}, {"entropy": None}, {"out": None}, {"stride": 99}, {"ostride": 99}, {"scale": 0.0},
                {"out": P, "ostride": 101}, {"lse": P + 2}, {"dl": P + 1}, {"de": P + 1}, {"out": 2 * P + 1}):
        assert back(**bad) == _lib.NTK_E_ARG, bad
    assert back(rows=0, x=None) == _lib.NTK_OK
