"""CPU-side checks of include/ntk_seq.h: every declared symbol is exported and bound, and bad arguments are refused
on the host, before any device call."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2206_08720_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2206_08720_amd.build import build
        build()
    return _lib.load()


def test_header_and_library_agree(lib):
    from paper_2206_08720_amd import _lib
    txt = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ntk_seq.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(ntk_[a-z_]+)\s*\(", txt))
    assert declared == set(_lib.EXPORTED_SEQ_SYMBOLS)
    assert all(hasattr(lib, n) for n in declared)


def _desc(**kw):
    from paper_2206_08720_amd import _lib
    d = dict(dtype=_lib.NTK_BF16, batch=2, q_len=8, k_len=64, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, softcap=0.0)
    d.update(kw)
    return _lib.ntk_attention_desc(**d)


@pytest.mark.parametrize("change,code", [
    ({"dtype": 3}, "NTK_E_ARG"), ({"batch": -1}, "NTK_E_ARG"), ({"q_len": -1}, "NTK_E_ARG"), ({"heads": 3}, "NTK_E_SHAPE"),
    ({"kv_heads": 0}, "NTK_E_SHAPE"), ({"head_dim": 0}, "NTK_E_ARG"), ({"head_dim": 129}, "NTK_E_UNSUPPORTED"),
    ({"scale": 0.0}, "NTK_E_ARG"), ({"scale": float("inf")}, "NTK_E_ARG"), ({"scale": float("nan")}, "NTK_E_ARG"),
    ({"softcap": -1.0}, "NTK_E_ARG"), ({"causal": 0, "prefix": 64}, "NTK_E_ARG"), ({"q_len": 1 << 30}, "NTK_E_UNSUPPORTED"),
    ({"k_len": (1 << 31) - 1}, "NTK_E_UNSUPPORTED"), ({"batch": 1 << 30, "kv_heads": 4}, "NTK_E_UNSUPPORTED")])
def test_attention_descriptor_refusals(lib, change, code):
    from paper_2206_08720_amd import _lib
    d = _desc(**change)
    assert lib.ntk_attention_workspace(ctypes.byref(d), 0) == getattr(_lib, code)
    assert "attention" in _lib.last_error()
    view = _lib.ntk_view(4096, 64, 64, 64)
    assert lib.ntk_attention(ctypes.byref(d), *[ctypes.byref(view)] * 4, None, None, 0, None) == getattr(_lib, code)
    assert lib.ntk_attention_bwd(ctypes.byref(d), *[ctypes.byref(view)] * 5, 4096, *[ctypes.byref(view)] * 3, None, 0, None) == getattr(_lib, code)


def test_attention_argument_refusals(lib):
    from paper_2206_08720_amd import _lib
    ok = ctypes.byref(_lib.ntk_view(4096, 64, 64, 64))
    d = ctypes.byref(_desc(q_len=1, k_len=4096))
    need = lib.ntk_attention_workspace(d, 0)
    assert need > 0
    for q in (None, ctypes.byref(_lib.ntk_view(0, 64, 64, 64)), ctypes.byref(_lib.ntk_view(4097, 64, 64, 64)),
              ctypes.byref(_lib.ntk_view(4096, 64, -64, 64))):
        assert lib.ntk_attention(d, q, ok, ok, ok, None, 4096, need, None) == _lib.NTK_E_ARG
    for work, size in ((None, need), (4096, need - 1), (4100, need)):
        assert lib.ntk_attention(d, ok, ok, ok, ok, None, work, size, None) == _lib.NTK_E_ARG
        assert "workspace" in _lib.last_error()
    assert lib.ntk_attention(d, ok, ok, ok, ok, 4097, 4096, need, None) == _lib.NTK_E_ARG
    need = lib.ntk_attention_workspace(d, 1)
    assert lib.ntk_attention_bwd(d, *[ok] * 5, None, *[ok] * 3, 4096, need, None) == _lib.NTK_E_ARG
    assert lib.ntk_attention_bwd(d, *[ok] * 5, 4096, *[ok] * 3, 4096, need - 1, None) == _lib.NTK_E_ARG
    assert lib.ntk_attention_bwd(d, *[ok] * 5, 4096, ok, None, ok, 4096, need, None) == _lib.NTK_E_ARG
    assert lib.ntk_attention(None, ok, ok, ok, ok, None, None, 0, None) == _lib.NTK_E_ARG


def test_norm_refusals(lib):
    from paper_2206_08720_amd import _lib
    P = 4096

    def norm(dtype=1, wtype=1, rows=4, width=64, x=P, xs=64, res=None, rs=0, w=P, eps=1e-6, y=P, h=None, scale=None):
        return lib.ntk_rms_norm(dtype, wtype, rows, width, x, xs, res, rs, w, eps, y, h, scale, None)

    for bad in ({"dtype": 5}, {"wtype": 2}, {"rows": -1}, {"width": 0}, {"x": None}, {"w": None}, {"y": None}, {"xs": 63},
                {"res": P, "rs": 1}, {"eps": -1.0}, {"eps": float("nan")}, {"x": P + 1}, {"h": P + 1}, {"scale": P + 2}):
        assert norm(**bad) == _lib.NTK_E_ARG, bad
    assert norm(width=32769, xs=40000) == _lib.NTK_E_UNSUPPORTED
    assert norm(rows=1 << 40) == _lib.NTK_E_UNSUPPORTED
    assert norm(rows=0, x=None) == _lib.NTK_OK
    assert lib.ntk_rms_norm_workspace(4, 0) == _lib.NTK_E_ARG
    need = lib.ntk_rms_norm_workspace(4, 64)
    args = [1, 1, 4, 64, P, 64, P, 64, P, None, 0, 1e-6, P, P, P, need, None]
    for at, value in ((4, None), (5, 3), (12, None), (13, None), (14, None), (15, need - 1), (14, P + 8)):
        assert lib.ntk_rms_norm_bwd(*args[:at], value, *args[at + 1:]) == _lib.NTK_E_ARG, at


def test_rotary_refusals(lib):
    from paper_2206_08720_amd import _lib
    ok = ctypes.byref(_lib.ntk_view(4096, 64, 64, 64))

    def rotary(dtype=1, b=2, n=3, h=4, hk=2, dim=64, rot=64, q=ok, k=ok, table=4096, max_pos=10, positions=None, first=0, qo=ok, ko=ok):
        return lib.ntk_rotary(dtype, b, n, h, hk, dim, rot, 0, 0, q, k, table, max_pos, positions, first, qo, ko, None)

    for bad in ({"dtype": -1}, {"b": -1}, {"dim": 0, "rot": 0}, {"q": None}, {"qo": None}, {"ko": None}, {"table": None}, {"max_pos": 0},
                {"first": -1}, {"positions": 4098}):
        assert rotary(**bad) in (_lib.NTK_E_ARG, _lib.NTK_E_SHAPE), bad
    for rot in (0, 63, 66):
        assert rotary(rot=rot) == _lib.NTK_E_SHAPE
    assert rotary(b=1 << 16, n=1 << 16) == _lib.NTK_E_UNSUPPORTED
    assert rotary(n=0) == _lib.NTK_OK
    s = _lib.ntk_rotary_scaling
    assert lib.ntk_rotary_table(0, 64, 1e4, None, 4096, None) == _lib.NTK_E_ARG
    assert lib.ntk_rotary_table(8, 64, 1.0, None, 4096, None) == _lib.NTK_E_ARG
    assert lib.ntk_rotary_table(8, 64, 1e4, None, None, None) == _lib.NTK_E_ARG
    for scaling in (s(9, 2.0, 1, 0, 1), s(1, 0.5, 1, 0, 1), s(3, 2.0, 0.0, 1, 32), s(3, 2.0, 8.0, 4, 4), s(2, float("nan"), 1, 0, 1)):
        assert lib.ntk_rotary_table(8, 64, 1e4, ctypes.byref(scaling), 4096, None) == _lib.NTK_E_ARG
