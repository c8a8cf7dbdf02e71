"""The rotation's kernels among each other: whichever sizes and alignment choose, a token's bits are
the same, in place or not, in a small call or a large one, alone or on the way into the pages."""
import pytest
import torch

import paper_2608_14191_amd as P
from paged_ref import TYPES

pytestmark = pytest.mark.gpu
D = 128


def _rope(rot, interleaved):
    freq = torch.from_numpy(P.aatc_rope_frequencies(rot, 500000.0)[0]).cuda()
    return freq, P.Rope(freq, P.ROPE_INTERLEAVED if interleaved else P.ROPE_HALF, 1.25)


def _turn(x, pos, freq, interleaved, inverse=False):
    """A few tokens [n][heads][D] rotated in 64 bits, and sum |a| + |b| of each channel's pair."""
    rot = 2 * freq.numel()
    lo, hi = ((slice(0, rot, 2), slice(1, rot, 2)) if interleaved
              else (slice(0, rot // 2), slice(rot // 2, rot)))
    angle = pos.double()[:, None] * freq
    c, s = 1.25 * angle.cos()[:, None], 1.25 * angle.sin()[:, None] * (-1 if inverse else 1)
    y, size = x.double(), x.double().abs()
    a, b = y[..., lo].clone(), y[..., hi].clone()
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    size[..., lo] = size[..., hi] = a.abs() + b.abs()
    return y, size


def _close(got, want, size, dtype):
    # half a step of the type; in fp32 below 8 2^-24 (|a| + |b|) factor, as for small calls
    fp32 = 8 * 2.0 ** -24 * 1.25 * size
    tiny = 2.0 ** -25 if dtype == torch.float16 else 1e-40
    assert torch.all((got.double() - want).abs() <= fp32 + torch.finfo(dtype).eps / 2 * (want.abs() + fp32) + tiny)


# Above 128 MiB of tokens rows of 16-byte pieces are moved past the caches.
@pytest.mark.parametrize("dtype,n,heads", [("bf16", 70001, 8), ("f16", 140003, 4), ("f32", 9001, 31)])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, False), (96, True), (50, True), (50, False)])
def test_rope_past_the_caches(dtype, n, heads, rot, interleaved):
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, heads, D, generator=g, device="cuda").to(TYPES[dtype])
    assert x.nbytes > 128 << 20
    pos = torch.randint(0, 10 ** 6, (n,), generator=g, device="cuda").int()
    freq, spec = _rope(rot, interleaved)
    stride, third = heads * D, n // 3 + 1
    for inverse in (False, True):
        out, pieces = torch.empty_like(x), torch.empty_like(x)
        P.aatc_rope(x, n, heads, stride, pos, spec, out, stride, inverse=inverse)
        for i in range(0, n, third):
            m = min(third, n - i)
            P.aatc_rope(x[i:], m, heads, stride, pos[i:], spec, pieces[i:], stride, inverse=inverse)
        assert torch.equal(out, pieces)
        again = x.clone()                                # in place
        P.aatc_rope(again, n, heads, stride, pos, spec, again, stride, inverse=inverse)
        assert torch.equal(again, out)
        some = torch.tensor([0, 1, n // 2, n - 1], device="cuda")
        _close(out[some], *_turn(x[some], pos[some], freq, interleaved, inverse), x.dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rot", [128, 96, 64, 50, 34, 2])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_bits_of_any_alignment(dtype, rot, interleaved, inverse):
    """Rows of 16-byte pieces and rows that begin an element behind one."""
    n, heads = 20011, 3
    g = torch.Generator(device="cuda").manual_seed(rot)
    x = torch.randn(n, heads, D, generator=g, device="cuda").to(TYPES[dtype])
    pos = torch.randint(-10 ** 6, 10 ** 6, (n,), generator=g, device="cuda").int()
    freq, spec = _rope(rot, interleaved)
    stride = heads * D
    out = torch.empty_like(x)
    P.aatc_rope(x, n, heads, stride, pos, spec, out, stride, inverse=inverse)
    _close(out, *_turn(x, pos, freq, interleaved, inverse), x.dtype)
    flat, odd = torch.zeros(1 + x.numel(), dtype=x.dtype, device="cuda"), torch.zeros(1 + x.numel(), dtype=x.dtype, device="cuda")
    flat[1:] = x.flatten()
    P.aatc_rope(flat[1:], n, heads, stride, pos, spec, odd[1:], stride, inverse=inverse)
    assert torch.equal(odd[1:].reshape(out.shape), out)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, True), (50, False), (50, True)])
def test_append_turns_as_rope_does(dtype, rot, interleaved):
    n, hq, hkv, page = 10007, 3, 2, 64
    g = torch.Generator(device="cuda").manual_seed(rot)
    x = torch.randn(n, hq + 2 * hkv, D, generator=g, device="cuda").to(TYPES[dtype])
    pos = torch.arange(n, device="cuda").int()
    pages = -(-n // page)
    table = torch.randperm(pages, generator=g, device="cuda").reshape(1, -1).int()
    pools = [torch.zeros(pages, hkv, page, D, dtype=x.dtype, device="cuda") for _ in range(2)]
    _, spec = _rope(rot, interleaved)
    stride = (hq + 2 * hkv) * D
    want = torch.empty_like(x)
    P.aatc_rope(x, n, hq + hkv, stride, pos, spec, want, stride)
    q_out = torch.empty(n, hq, D, dtype=x.dtype, device="cuda")
    P.aatc_paged_append(P.PagedCache(*pools), table, n, x[:, hq:hq + hkv], x[:, hq + hkv:], stride, stride,
                        torch.zeros(n, device="cuda").int(), pos, rope=spec, n_q_heads=hq, q=x[:, :hq],
                        q_tok_stride=stride, q_out=q_out, q_out_tok_stride=hq * D)
    assert torch.equal(q_out, want[:, :hq])
    assert torch.equal(pools[0][table[0].long()].transpose(1, 2).reshape(-1, hkv, D)[:n], want[:, hq:hq + hkv])
