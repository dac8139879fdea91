"""The example that runs the sequence operators together (examples/sequence_ntk.py): its trunk's gradients
against torch's in 64 bits, its token pass against the whole one, and the loss it lowers."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("sequence_ntk", os.path.join(ROOT, "examples", "sequence_ntk.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _reference(trunk, weights, x, docs):
    """The trunk in 64 bits from elementary operations."""
    import torch
    norm_in, qkv, out, norm_out = weights
    B, n, _ = x.shape

    def norm(t, w):
        return t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w

    parts = (norm(x, norm_in) @ qkv.T).view(B, n, -1, trunk.dim)
    q, k, v = parts.split((trunk.heads, trunk.kv_heads, trunk.kv_heads), 2)
    c, s = trunk.table.cpu().double()[:n, None, :, 0], trunk.table.cpu().double()[:n, None, :, 1]
    half = trunk.dim // 2

    def turn(t):
        u, w = t[..., :half], t[..., half:]
        return torch.cat((u * c - w * s, w * c + u * s), -1)

    grp = trunk.heads // trunk.kv_heads
    q, k, v = turn(q).transpose(1, 2), turn(k).transpose(1, 2).repeat_interleave(grp, 1), v.transpose(1, 2).repeat_interleave(grp, 1)
    z = trunk.softcap * torch.tanh(q @ k.transpose(2, 3) * trunk.dim ** -0.5 / trunk.softcap)
    seen = (torch.arange(n)[:, None] >= torch.arange(n)) & (docs[:, None, :, None] == docs[:, None, None, :])
    a = torch.softmax(z.masked_fill(~seen, float("-inf")), -1) @ v
    return norm(a.transpose(1, 2).flatten(2) @ out.T + x, norm_out)


def test_trunk_gradients_and_features():
    """fp32 trunk: every factor of the chain is good to about 2e-6 of its norm (products of up to 512 terms in fp32);
    a dozen of them in a row, taken in norm: 5e-5."""
    import torch
    m = _example()
    trunk = m.Trunk(96, 4, 2, 32, 60, torch.float32, softcap=5.0)
    g = torch.Generator().manual_seed(3)
    x, dz = (torch.randn(3, 50, 96, generator=g) for _ in range(2))
    docs = torch.tensor([j // 20 for j in range(50)], dtype=torch.int32).expand(3, 50).contiguous()
    z, saved = trunk.forward(x.cuda(), docs.cuda())
    got = trunk.backward(dz.cuda(), saved)
    w = [t.cpu().double().requires_grad_() for t in trunk.weights()]
    ref = _reference(trunk, w, x.double(), docs)
    grads = torch.autograd.grad(ref, w, dz.double())
    for a, b in zip([z] + got, [ref.detach()] + list(grads)):
        assert float((a.cpu().double() - b).norm() / b.norm()) <= 5e-5


def test_example_runs():
    """The whole example in fp32 and bf16: the loss falls, Theta is finite and changes, and the token pass gives the whole
    pass's features (fp32 to 5e-5 of their norm, bf16 to a dozen roundings of 2^-8 in a row, 3e-2)."""
    import torch
    m = _example()
    for dtype, tol in ((torch.float32, 5e-5), (torch.bfloat16, 3e-2)):
        thetas, losses, features, answer = m.main(batch=5, length=70, width=64, heads=4, kv_heads=2, dim=32, steps=2, dtype=dtype, quiet=True)
        assert losses[2] < losses[0]
        assert all(torch.isfinite(t).all() for t in thetas) and not torch.equal(thetas[0], thetas[2])
        assert float((answer - features).norm() / features.norm()) <= tol
