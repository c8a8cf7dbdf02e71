"""aatc_rope and aatc_paged_append against the 64-bit rotation."""
import pytest
import torch

import paper_2608_14191_amd as P
from paged_ref import HALF_STEP, TYPES, pool, to_cuda, turn

pytestmark = pytest.mark.gpu
D = 128


def _spec(rot, interleaved, factor=1.0):
    freq = torch.from_numpy(P.aatc_rope_frequencies(rot, 500000.0)[0])
    return freq, P.Rope(freq.cuda(), P.ROPE_INTERLEAVED if interleaved else P.ROPE_HALF, factor)


def _bound(x, rot, want, dtype, interleaved, factor=1.0):
    """Half a step of the output's type, and in fp32: the angle's rest to 2^-24 of half a turn
    (pi 2^-24), sine and cosine to 2 ulps, two products and a sum: below 8 2^-24 (|a| + |b|)."""
    a = x.double().abs()
    pair = a.clone()
    lo, hi = ((slice(0, rot, 2), slice(1, rot, 2)) if interleaved
              else (slice(0, rot // 2), slice(rot // 2, rot)))
    pair[..., lo] = pair[..., hi] = a[..., lo] + a[..., hi]
    fp32 = 8 * 2.0 ** -24 * pair * factor
    # (f16 below 2^-14: half of its smallest step)
    tiny = 2.0 ** -25 if dtype == torch.float16 else 1e-40
    return fp32 + HALF_STEP[dtype] * (want.abs() + fp32) + tiny


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rot", [128, 96, 64, 50, 16, 2])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_types_and_parts(dtype, rot, interleaved):
    g = torch.Generator().manual_seed(rot)
    n, heads = 37, 5
    x = torch.randn(n, heads, D, generator=g).to(TYPES[dtype])
    pos = torch.randint(-10 ** 6, 10 ** 6, (n,), generator=g).int()
    pos[0], pos[1] = 0, 2 ** 31 - 1
    freq, spec = _spec(rot, interleaved, 1.25)
    for inverse in (False, True):
        out = torch.empty_like(x, device="cuda")
        P.aatc_rope(x.cuda(), n, heads, heads * D, pos.cuda(), spec, out, heads * D, inverse=inverse)
        want = turn(x, pos, freq, 1.25, interleaved, inverse)
        got = out.cpu()
        assert torch.all((got.double() - want).abs() <= _bound(x, rot, want, x.dtype, interleaved, 1.25))
        assert torch.equal(got[..., rot:], x[..., rot:])
        again = x.cuda()                             # in place
        P.aatc_rope(again, n, heads, heads * D, pos.cuda(), spec, again, heads * D, inverse=inverse)
        assert torch.equal(again.cpu(), got)


@pytest.mark.parametrize("n,heads", [(1, 1), (1, 64), (3, 28), (1000, 8), (5, 200)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_sizes(n, heads, interleaved):
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, heads, D, generator=g).to(torch.bfloat16)
    pos = torch.randint(0, 200000, (n,), generator=g).int()
    freq, spec = _spec(D, interleaved)
    out = torch.empty_like(x, device="cuda")
    P.aatc_rope(x.cuda(), n, heads, heads * D, pos.cuda(), spec, out, heads * D)
    want = turn(x, pos, freq, 1.0, interleaved)
    assert torch.all((out.cpu().double() - want).abs() <= _bound(x, D, want, x.dtype, interleaved))


@pytest.mark.parametrize("offset,pad", [(0, 24), (1, 0), (4, 3), (8, 8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_strides_and_alignment(offset, pad, dtype, interleaved):
    """Token strides and starts of any alignment: the same bits; what lies between stays."""
    g = torch.Generator().manual_seed(3)
    n, heads = 11, 3
    x = torch.randn(n, heads, D, generator=g).to(TYPES[dtype])
    pos = torch.arange(n).int() * 1001
    freq, spec = _spec(96, interleaved)
    out = torch.empty_like(x, device="cuda")
    P.aatc_rope(x.cuda(), n, heads, heads * D, pos.cuda(), spec, out, heads * D)
    stride = heads * D + pad
    flat = torch.zeros(offset + n * stride, dtype=x.dtype)
    view = flat[offset:].reshape(n, stride)
    view[:, :heads * D] = x.reshape(n, -1)
    src = flat.cuda()
    dst = torch.full_like(src, 7.0)
    P.aatc_rope(src[offset:], n, heads, stride, pos.cuda(), spec, dst[offset:], stride)
    got = dst.cpu()[offset:].reshape(n, stride)
    assert torch.equal(got[:, :heads * D].reshape(n, heads, D), out.cpu())
    assert torch.all(got[:, heads * D:] == 7.0) and torch.all(dst[:offset] == 7.0)


def test_rope_gradient():
    """The inverse is the gradient: <dy, R x> differs by <R^T dy, dx>; and by differences."""
    g = torch.Generator().manual_seed(8)
    n, heads = 9, 2
    x, dy, dx = (torch.randn(n, heads, D, generator=g) for _ in range(3))
    pos = torch.randint(0, 10 ** 5, (n,), generator=g).int().cuda()
    _, spec = _spec(64, False, 1.3)

    def run(v, inverse=False):
        out = torch.empty(n, heads, D, device="cuda")
        P.aatc_rope(v.float().cuda(), n, heads, heads * D, pos, spec, out, heads * D, inverse=inverse)
        return out.cpu().double()
    grad = run(dy, inverse=True)
    # linear: the difference quotient is exact but for rounding, 2^-22 of the terms' sizes
    change = (dy.double() * (run(x + dx) - run(x))).sum()
    assert abs(change - (grad * dx.double()).sum()) <= 2.0 ** -20 * (dy.double().abs() * 4 * (x.abs() + dx.abs()).double()).sum()
    rows = torch.eye(D).reshape(D, 1, D).expand(D, 1, D)
    jac = torch.empty(D, 1, D, device="cuda")
    p = torch.full((D,), 777, dtype=torch.int32, device="cuda")
    P.aatc_rope(rows.contiguous().cuda(), D, 1, D, p, spec, jac, D)
    back = torch.empty_like(jac)
    P.aatc_rope(rows.contiguous().cuda(), D, 1, D, p, spec, back, D, inverse=True)
    assert torch.equal(jac[:, 0].cpu(), back[:, 0].cpu().T)


# ------------------------------------------------------------------------------- append
def _append_case(seed, tokens, rows, hq, hkv, page, x="bf16", cache="bf16", order="head"):
    g = torch.Generator().manual_seed(seed)
    per_row = 6
    n_pages = rows * per_row + 2
    table = torch.randperm(n_pages, generator=g)[:rows * per_row].reshape(rows, per_row).int()
    slots = torch.randperm(rows * per_row * page, generator=g)[:tokens]
    seq, pos = (slots // (per_row * page)).int(), (slots % (per_row * page)).int()
    qkv = torch.randn(tokens, hq + 2 * hkv, D, generator=g).to(TYPES[x])
    pools = [pool(g, n_pages, hkv, page, TYPES[cache], order) for _ in range(2)]
    return table, seq, pos, qkv, pools


def _append(table, seq, pos, qkv, pools, hq, hkv, spec, in_place=False):
    n, stride = qkv.shape[0], qkv.shape[1] * D
    dev = qkv.cuda()
    kp, vp = (to_cuda(p) for p in pools)
    q_out = dev[:, :hq] if in_place else torch.full((n, hq, D), 9.0, dtype=qkv.dtype, device="cuda")
    P.aatc_paged_append(P.PagedCache(kp, vp), table.cuda(), n, dev[:, hq:hq + hkv], dev[:, hq + hkv:],
                        stride, stride, None if seq is None else seq.cuda(), pos.cuda(), rope=spec,
                        n_q_heads=hq, q=dev[:, :hq] if hq else None, q_tok_stride=stride,
                        q_out=q_out if hq else None,
                        q_out_tok_stride=stride if in_place else hq * D)
    torch.cuda.synchronize()
    return q_out.cpu(), kp.cpu(), vp.cpu()


@pytest.mark.parametrize("x,cache", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f16"),
                                     ("bf16", "f32"), ("f16", "f16"), ("f32", "f32"),
                                     ("f16", "bf16"), ("bf16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, True), (50, False), (0, False)])
def test_append(x, cache, order, rot, interleaved):
    hq, hkv, page, n = 6, 2, 16, 53
    table, seq, pos, qkv, pools = _append_case(rot, n, 5, hq, hkv, page, x, cache, order)
    pos[3] = pos[10] = -1                            # padding
    seq[20], seq[21] = -1, 5                         # no such sequence
    pos[22] = 6 * page                               # no such page
    table[int(seq[30]), int(pos[30]) // page] = -1   # a page that is not there
    freq, spec = _spec(rot, interleaved, 1.1) if rot else (torch.zeros(0), None)
    factor = 1.1 if rot else 1.0
    q, k, v = _append(table, seq, pos, qkv, pools, hq, hkv, spec)
    want_q = turn(qkv[:, :hq], pos, freq, factor, interleaved)
    want_k = turn(qkv[:, hq:hq + hkv], pos, freq, factor, interleaved)
    kept = [p.clone() for p in pools]
    for t in range(n):
        if pos[t] < 0:
            assert torch.all(q[t] == 9.0)
            continue
        err = (q[t].double() - want_q[t]).abs()
        assert torch.all(err <= _bound(qkv[t, :hq], rot, want_q[t], qkv.dtype, interleaved, factor))
        if not (0 <= seq[t] < 5) or pos[t] >= 6 * page:
            continue
        at, slot = int(table[seq[t], pos[t] // page]), int(pos[t]) % page
        if at < 0:
            continue
        err = (k[at, :, slot].double() - want_k[t]).abs()
        assert torch.all(err <= _bound(qkv[t, hq:hq + hkv], rot, want_k[t], TYPES[cache],
                                       interleaved, factor))
        assert torch.equal(v[at, :, slot], qkv[t, hq + hkv:].to(TYPES[cache]))
        kept[0][at, :, slot], kept[1][at, :, slot] = k[at, :, slot], v[at, :, slot]
    assert torch.equal(k, kept[0]) and torch.equal(v, kept[1])     # nothing else was touched


def test_append_one_token_per_sequence_in_place():
    hq, hkv, page = 8, 2, 8
    table, _, _, qkv, pools = _append_case(4, 5, 5, hq, hkv, page)
    pos = torch.tensor([0, 7, 8, 47, 23]).int()
    freq, spec = _spec(128, False)
    a = _append(table, torch.arange(5).int(), pos, qkv, pools, hq, hkv, spec)
    b = _append(table, None, pos, qkv, pools, hq, hkv, spec, in_place=True)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    c = _append(table, None, pos, qkv[:, hq:], pools, 0, hkv, spec)      # no queries
    assert torch.equal(c[1], a[1]) and torch.equal(c[2], a[2])


def test_append_keeps_bits_of_what_is_not_rotated():
    """Channels behind rot and values keep their bits, NaN payloads among them."""
    bits = torch.randint(-2 ** 15, 2 ** 15 - 1, (4, 3, D), generator=torch.Generator().manual_seed(1))
    qkv = bits.to(torch.int16).view(torch.bfloat16)
    table = torch.zeros(1, 1).int()
    _, spec = _spec(16, False)
    pools = [torch.zeros(1, 1, 8, D, dtype=torch.bfloat16) for _ in range(2)]
    q, _, _ = _append(table, torch.zeros(4).int(), torch.arange(4).int(), qkv, pools, 1, 1, spec)
    assert torch.equal(q[..., 16:].view(torch.int16), qkv[:, :1, 16:].view(torch.int16))
