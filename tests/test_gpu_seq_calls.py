"""Calls of the sequence operators' binding that it refuses, or answers, on the GPU."""
import pytest

from tests.test_gpu_seq import _close, _norm_reference, _oracle, _rand

pytestmark = pytest.mark.gpu


def test_rows_past_2_to_the_24():
    """Narrow rows in their millions, and caches of 2^26 keys in all: each launch holds them."""
    import torch
    from paper_2206_08720_amd import seq
    rows = 2 ** 24 + 5
    x, w = torch.randn(rows, 8, device="cuda").bfloat16(), torch.ones(8, dtype=torch.bfloat16, device="cuda")
    y = seq.rms_norm(x, w)
    dx, _ = seq.rms_norm_backward(x, x, w)
    for part in (slice(0, 3), slice(rows - 3, rows)):
        a = x[part].cpu()
        ref = _norm_reference(a, None, w.cpu(), 1e-6, "bf16", a, None, a)
        _close("y", y[part], *ref["y"])
        _close("dx", dx[part], *ref["dx"])
    table = seq.rotary_table(8, 2)
    q = x[:, :2].reshape(1, rows, 1, 2).contiguous()
    at = (torch.arange(rows, device="cuda") % 8).int()[None]
    t = seq.rotary(q, table, at)
    assert torch.equal(t[:, -9:], seq.rotary(q[:, -9:].contiguous(), table, at[:, -9:].contiguous()))
    b, n = 2048, 4099
    kc, vc, q = (_rand((4, m, h, 8), 860 + i, "bf16") for i, (m, h) in enumerate(((n, 8), (n, 8), (1, 8))))
    o = seq.attention(q.cuda().repeat(b // 4, 1, 1, 1), kc.cuda().repeat(b // 4, 1, 1, 1), vc.cuda().repeat(b // 4, 1, 1, 1))
    ref = _oracle(q, kc, vc, "bf16")["o"]
    _close("o", o[:4], *ref)
    _close("o", o[-4:], *ref)
