"""The NTK of a head on a sequence trunk's features, while the trunk is trained.

A trunk of one block (norm, attention with rotary positions, residual, norm) reads packed token embeddings; the
features of each sequence's last position are the inputs X of a small fully-connected head, whose
Theta(X, X) the library computes.  Between two NTKs the trunk takes gradient steps towards target
features, its backward pass made of the operators' own; at the end it reads the sequences token by token
over a cache of keys and values.

    python examples/sequence_ntk.py        # on an MI355X, after the library is built
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import workloads as wl  # noqa: E402
from paper_2206_08720_amd import seq  # noqa: E402
from paper_2206_08720_amd.ntk import NTK  # noqa: E402


class Trunk:
    """One block; products with the weights are torch's, everything else is `seq`."""

    def __init__(self, width, heads, kv_heads, dim, max_pos, dtype, seed=0, softcap=30.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.softcap = heads, kv_heads, dim, softcap
        parts = heads + 2 * kv_heads

        def weight(out, inp):
            return (torch.randn(out, inp, device="cuda", generator=g) * inp ** -0.5).to(dtype)

        self.norm_in, self.norm_out = (torch.ones(width, device="cuda", dtype=dtype) for _ in range(2))
        self.qkv, self.out = weight(parts * dim, width), weight(width, heads * dim)
        self.table = seq.rotary_table(max_pos, dim)

    def weights(self):
        return [self.norm_in, self.qkv, self.out, self.norm_out]

    def _split(self, y):
        b, n = y.shape[:2]
        return (y @ self.qkv.T).view(b, n, -1, self.dim).split((self.heads, self.kv_heads, self.kv_heads), 2)

    def forward(self, x, docs=None):
        """z [batch, length, width] for x of the same shape, and what the backward pass reads."""
        y = seq.rms_norm(x, self.norm_in)
        q, k, v = self._split(y)
        q, k = seq.rotary(q, self.table, k=k)
        a, lse = seq.attention(q, k, v, causal=True, softcap=self.softcap, docs=docs, return_lse=True)
        z, h = seq.rms_norm(a.flatten(2) @ self.out.T, self.norm_out, residual=x)
        return z, (x, y, q, k, v, a, lse, h, docs)

    def backward(self, dz, saved):
        """Gradients of weights()."""
        x, y, q, k, v, a, lse, h, docs = saved
        d, d_norm_out = seq.rms_norm_backward(dz, h, self.norm_out)
        d_out = d.flatten(0, 1).T @ a.flatten(2).flatten(0, 1)
        da = (d @ self.out).view(a.shape)
        dq, dk, dv = seq.attention_backward(da, q, k, v, a, lse, causal=True, softcap=self.softcap, docs=docs)
        dq, dk = seq.rotary(dq, self.table, k=dk, inverse=True)
        dqkv = torch.cat((dq, dk, dv), 2).flatten(2)
        d_qkv = dqkv.flatten(0, 1).T @ y.flatten(0, 1)
        _, d_norm_in = seq.rms_norm_backward(dqkv @ self.qkv, x, self.norm_in)
        return [d_norm_in, d_qkv, d_out, d_norm_out]

    def token(self, x, cache, lens):
        """z of the next position of every sequence: x [batch, 1, width]; cache [2, batch, capacity, kv_heads, dim] holds
        lens[b] positions and gets one more."""
        y = seq.rms_norm(x, self.norm_in)
        q, k, v = self._split(y)
        at = lens[:, None].contiguous()
        q, k = seq.rotary(q, self.table, at, k=k)
        rows = torch.arange(len(lens), device="cuda")
        cache[0][rows, lens.long()], cache[1][rows, lens.long()] = k[:, 0], v[:, 0]
        a = seq.attention(q, cache[0], cache[1], causal=True, softcap=self.softcap, k_lens=lens + 1)
        return seq.rms_norm(a.flatten(2) @ self.out.T, self.norm_out, residual=x)[0]


def main(batch=16, length=200, width=256, heads=8, kv_heads=2, dim=64, steps=3, dtype=torch.bfloat16, quiet=False):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(batch, length, width, device="cuda", generator=g).to(dtype)
    target = torch.randn(batch, width, device="cuda", generator=g)
    # two documents a row: the features are those of the second
    docs = (torch.arange(length, device="cuda") >= length // 3).int().expand(batch, length).contiguous()
    trunk = Trunk(width, heads, kv_heads, dim, length, dtype)
    spec = wl.fcn_spec("head", width, [128], 4, act="erf", bias=True)
    head = [torch.from_numpy(p).cuda() for p in wl.make_params(spec, 7)]
    ntk = NTK(spec, batch, batch)
    thetas, losses = [], []
    try:
        for step in range(steps + 1):
            z, saved = trunk.forward(x, docs)
            features = z[:, -1].float().contiguous()
            thetas.append(ntk.compute(head, features))
            losses.append(0.5 * float((features - target).square().sum(1).mean()))
            if not quiet:
                eig = torch.linalg.eigvalsh(thetas[-1].permute(0, 2, 1, 3).reshape(batch * 4, batch * 4).double().cpu())
                print(f"step {step}: loss {losses[-1]:.4f}, Theta's largest eigenvalue {float(eig[-1]):.3f}, smallest {float(eig[0]):.3e}",
                      flush=True)
            if step < steps:
                dz = torch.zeros_like(z)
                dz[:, -1] = ((features - target) / batch).to(dtype)
                for w, dw in zip(trunk.weights(), trunk.backward(dz, saved)):
                    w.sub_((0.1 * dw.float()).to(dtype))
    finally:
        ntk.close()
    # the second document again, token by token; its positions start over, which rotary's relative angles do not see
    first = length // 3
    cache = torch.zeros(2, batch, length - first, kv_heads, dim, device="cuda", dtype=dtype)
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    for t in range(first, length):
        out = trunk.token(x[:, t:t + 1], cache, lens)
        lens += 1
    answer = out[:, 0].float()
    if not quiet:
        print(f"token by token against the whole pass: largest difference {float((answer - features).abs().max()):.2e}")
    return thetas, losses, features, answer


if __name__ == "__main__":
    main()
