"""The sequence operators' limits (include/ntk_seq.h), on the host: what a launch holds is refused by that launch alone."""
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


def _workspace(lib, backward, **kw):
    from paper_2206_08720_amd import _lib
    d = dict(dtype=_lib.NTK_BF16, batch=2, q_len=8, k_len=64, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, softcap=0.0)
    d.update(kw)
    return lib.ntk_attention_workspace(ctypes.byref(_lib.ntk_attention_desc(**d)), backward)


def test_tokens_over_large_caches(lib):
    """512 sequences of 8 heads and 32768 places: 2^27 keys, in one launch of 4096 workgroups."""
    assert _workspace(lib, 0, batch=512, q_len=1, k_len=32768, heads=32, kv_heads=8, head_dim=128) >= 0


def test_rows_of_large_training_batches(lib):
    """2^27 rows of 16 a workgroup, 2^20 tiles."""
    sizes = dict(batch=64, q_len=65536, k_len=65536, heads=32, kv_heads=32, head_dim=64)
    assert _workspace(lib, 0, **sizes) >= 0 and _workspace(lib, 1, **sizes) >= 0


def test_what_one_launch_does_not_hold(lib):
    from paper_2206_08720_amd import _lib
    for backward in (0, 1):
        assert _workspace(lib, backward, batch=1 << 14, q_len=1 << 18, k_len=1 << 18, heads=8, kv_heads=8) == _lib.NTK_E_UNSUPPORTED


def test_rotary_heads_past_32_bits(lib):
    """2^30 heads of q and as many of k: their sum is counted in 64 bits."""
    from paper_2206_08720_amd import _lib
    v = ctypes.byref(_lib.ntk_view(4096, 0, 0, 0))
    for q, k in ((1 << 30, 1 << 30), (2147483647, 2147483647), (1 << 30, 0), (1 << 20, 1)):
        assert lib.ntk_rotary(1, 1, 1, q, k, 64, 64, 0, 0, v, v, 4096, 8, None, 0, v, v, None) == _lib.NTK_E_UNSUPPORTED


def test_outputs_that_overlap(lib):
    """Rows of an output over each other, or an output that starts where an operand does."""
    from paper_2206_08720_amd import _lib
    d = _lib.ntk_attention_desc(_lib.NTK_BF16, 2, 8, 64, 4, 2, 64, 1, 0.125, 0.0)

    def view(place, b=1 << 20, n=256, h=64):
        return ctypes.byref(_lib.ntk_view(4096 * place, b, n, h))

    q, k, v, o = (view(i + 1) for i in range(4))
    need = [lib.ntk_attention_workspace(ctypes.byref(d), i) for i in (0, 1)]
    for out in (q, k, v, view(9, b=0), view(9, n=0), view(9, h=0), view(9, n=63)):
        assert lib.ntk_attention(ctypes.byref(d), q, k, v, out, None, 4096, need[0], None) == _lib.NTK_E_ARG
        assert "overlaps" in _lib.last_error()
        for at in range(3):
            grads = [view(10 + i) for i in range(3)]
            grads[at] = out
            assert lib.ntk_attention_bwd(ctypes.byref(d), view(8), q, k, v, o, 4096, *grads, 4096, need[1], None) == _lib.NTK_E_ARG
            assert "overlaps" in _lib.last_error()
    grads = [view(10), view(11), view(11)]
    assert lib.ntk_attention_bwd(ctypes.byref(d), view(8), q, k, v, o, 4096, *grads, 4096, need[1], None) == _lib.NTK_E_ARG
    for qo, ko in ((view(9, n=0), view(10)), (view(9), view(10, h=0)), (view(9), view(9)), (k, view(9)), (view(9), q)):
        assert lib.ntk_rotary(1, 2, 8, 4, 2, 64, 64, 0, 0, q, k, 4096, 8, None, 0, qo, ko, None) == _lib.NTK_E_ARG
        assert "overlaps" in _lib.last_error()


def test_scores_constants_in_range(lib):
    """scale log2(e), softcap log2(e) and their quotient are formed in fp32: inf times a raw score of 0 would be NaN."""
    from paper_2206_08720_amd import _lib
    for bad in (dict(scale=3e38), dict(softcap=3e38), dict(softcap=1e-40), dict(scale=1e30, softcap=1e-30)):
        for backward in (0, 1):
            assert _workspace(lib, backward, **bad) == _lib.NTK_E_ARG
    for good in (dict(scale=2e38), dict(softcap=2e38), dict(softcap=1e-37), dict(scale=1e-40)):
        assert _workspace(lib, 0, **good) >= 0


def test_the_table_goes_to_the_current_gpu(monkeypatch):
    import torch
    from paper_2206_08720_amd import seq
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    for device in (None, "cuda", torch.device("cuda")):
        assert seq._gpu(device) == torch.device("cuda", 3)
    assert seq._gpu("cuda:1") == torch.device("cuda", 1) and seq._gpu(torch.device("cuda", 0)).index == 0
    with pytest.raises(ValueError):
        seq._gpu("cpu")
