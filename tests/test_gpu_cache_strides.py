"""The cache in pages where its parts lie far apart (paper_2206_08720_amd.seq): slots outermost in memory, and pages past 2^32 bytes in 8
bits.  Tolerances as in tests/test_gpu_cache.py."""
import pytest

from tests.test_gpu_cache import _ints
from tests.test_gpu_seq import _close, _oracle, _rand

pytestmark = pytest.mark.gpu


def _apart(e4m3, pages, size, heads, dim, slot_bytes, at=0):
    """A cache whose slots lie `slot_bytes` apart, pages and heads within; k and v share the memory, v behind k's cells.  What lies
    between is left as it came, but for the places that a slot distance cut to 32 bits would name."""
    import torch
    from paper_2206_08720_amd import seq
    kind = torch.uint8 if e4m3 else torch.bfloat16
    step, row = slot_bytes // kind.itemsize, heads * dim
    whole = torch.empty(at + step * (size - 1) + 2 * pages * row, dtype=kind, device="cuda")
    whole[:at + 4 * pages * row * size].fill_(0x30 if e4m3 else 3.0)
    k, v = (whole.as_strided((pages, size, heads, dim), (row, step, dim, 1), at + i * pages * row) for i in range(2))
    scales = [torch.ones(pages, heads, device="cuda") for _ in range(2)] if e4m3 else [None, None]
    if e4m3:
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    return seq.PagedCache(k, v, *scales)


def _through(cache, table, n, Hk, D, e4m3):
    """Appends n tokens to each sequence, reads them for a prompt and for a token, and checks cells and results."""
    import torch
    from paper_2206_08720_amd import seq
    B, size = table.shape[0], cache.k.shape[1]
    x = _rand((B, n, 2 * Hk, D), 20, "bf16")
    kk, vv = x.cuda().split((Hk, Hk), 2)
    seq.cache_append(cache, table.cuda(), _ints([0] * B), kk, vv)
    q = _rand((B, n, 2 * Hk, D), 21, "bf16")
    lens = _ints([n] * B)
    o = seq.attention_cached(q.cuda(), cache, table.cuda(), lens)
    one = seq.attention_cached(q[:, -1:].cuda(), cache, table.cuda(), lens)
    for b in range(B):
        got = []
        for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
            got.append(torch.stack([t[int(table[b, p // size]), p % size].cpu().double() * (1 if s is None else s[int(table[b, p // size])].cpu().double()[:, None])
                                    for p in range(n)]))
        # 2^-4 of the value and half the smallest step, 2^-10 times a scale of at most 2^-6 (values below 448 / 64)
        limit = 2.0 ** -4 * x[b].double().abs() + 2.0 ** -16 if e4m3 else 0.0 * x[b].double()
        assert ((torch.cat(got, 1) - x[b].double()).abs() <= limit).all()
        ref = _oracle(q[b:b + 1], got[0][None], got[1][None], "bf16", causal=True)
        _close("o", o[b:b + 1], *ref["o"])
        _close("one", one[b:b + 1], ref["o"][0][:, -1:], ref["o"][1][:, -1:])


@pytest.mark.parametrize("slot_bytes", [(1 << 32) + 256, 1 << 32], ids=["past-2^32", "at-2^32"])
@pytest.mark.parametrize("e4m3", [False, True])
def test_slots_past_32_bits(e4m3, slot_bytes):
    """28 GiB with the slots of a page outermost, their distance 2^32 bytes and a little more."""
    import torch
    cache = _apart(e4m3, 6, 8, 2, 64, slot_bytes)
    _through(cache, torch.tensor([[5, 0, 3], [1, 4, 2]]).int(), 21, 2, 64, e4m3)
    del cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("e4m3", [False, True])
def test_slots_past_an_offset_within_a_page(e4m3):
    """Slots of 32 bits' distance, the last of a page past 2^31 bytes from its first."""
    import torch
    cache = _apart(e4m3, 4, 64, 2, 128, (1 << 25) + 4096)
    _through(cache, torch.tensor([[3, 0], [2, 1]]).int(), 70, 2, 128, e4m3)
    del cache
    torch.cuda.empty_cache()


def test_pages_past_32_bits_of_bytes():
    """8 bits: over 4 GiB of pages in each array, the last of them in use."""
    import torch
    from paper_2206_08720_amd import seq
    pages, size, Hk, D = (1 << 19) + 9, 16, 4, 128
    assert pages * size * Hk * D > 1 << 32
    k, v = (torch.empty(pages, Hk, size, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).transpose(1, 2) for _ in range(2))
    cache = seq.PagedCache(k, v, *(torch.ones(pages, Hk, device="cuda") for _ in range(2)))
    _through(cache, torch.tensor([[pages - 1, 3, pages - 2], [0, pages - 5, 7]]).int(), 40, Hk, D, True)
    del k, v, cache
    torch.cuda.empty_cache()
