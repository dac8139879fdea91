"""CPU check of how many workgroups share the attention over a long cache: as many as run at once, which the workspace shows."""
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


COMPUTE_UNITS, LDS = 256, 160 << 10


@pytest.mark.parametrize("dim", [32, 64, 80, 128])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_tokens_of_long_caches(lib, dtype, e4m3, dim):
    """A workgroup of 2 or 4 waves holds 32 keys and values a wave in the queries' type, in 16 and 32 bits twice (the next ones are on their
    way), and two of them run on a compute unit where its LDS (and the registers) hold both: those are the workers, each with two
    partial results of 32 rows."""
    from paper_2206_08720_amd import _lib
    code = {"f32": _lib.NTK_F32, "bf16": _lib.NTK_BF16, "f16": _lib.NTK_F16}[dtype]
    size, padded = (4 if dtype == "f32" else 2), (64 if dim <= 64 else 128)
    desc = _lib.ntk_attention_desc(code, 16, 1, 1 << 17, 8, 8, dim, 1, 0.125, 0.0, 4096)
    got = lib.ntk_attention_cached_workspace(ctypes.byref(desc), _lib.NTK_E4M3 if e4m3 else code)
    wave = 2 * 32 * padded * size * (1 if e4m3 else 2)
    group = wave * (4 if 4 * wave <= 128 << 10 else 2)
    workers = COMPUTE_UNITS * (2 if 2 * group <= LDS else 1)
    assert got == 4 * workers * (2 * 32 * (padded + 2) + 4)
