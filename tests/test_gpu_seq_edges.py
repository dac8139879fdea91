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
