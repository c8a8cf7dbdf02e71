"""The paged operators where sizes choose another kernel: tokens, pools and copies too large for the
caches, and more tokens than one launch takes.  The same bits as in smaller pieces, and the formula."""
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


def test_rope_of_more_tokens_than_a_launch():
    """2^25 tokens a launch."""
    n = (1 << 25) + 5
    x = torch.randn(n // 8 + 1, D, device="cuda", dtype=torch.bfloat16).repeat(8, 1)[:n]
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    freq, spec = _rope(128, False)
    out = torch.zeros_like(x)
    P.aatc_rope(x, n, 1, D, pos, spec, out, D)
    some = torch.tensor([0, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, n - 1], device="cuda")
    _close(out[some][:, None], *_turn(x[some][:, None], pos[some], freq, False), x.dtype)
    half = n // 2 + 3
    pieces = torch.zeros_like(x)
    for i in (0, half):
        P.aatc_rope(x[i:], min(half, n - i), 1, D, pos[i:], spec, pieces[i:], D)
    assert torch.equal(out, pieces)


@pytest.mark.parametrize("x,cache", [("f32", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (96, True)])
def test_append_past_the_caches(x, cache, order, rot, interleaved):
    hq, hkv, page = 28, 4, 64
    heads = hq + 2 * hkv
    n = (128 << 20) // (heads * D * (4 if x == "f32" else 2)) + 77
    rows, per_row = 3, -(-n // (3 * page)) + 1
    g = torch.Generator(device="cuda").manual_seed(n)
    qkv = torch.randn(n, heads, D, generator=g, device="cuda").to(TYPES[x])
    seq = (torch.arange(n, device="cuda") % rows).int()
    pos = (torch.arange(n, device="cuda") // rows).int()
    pos[100:120] = -1
    table = torch.randperm(rows * per_row + 2, generator=g, device="cuda")[:rows * per_row].reshape(rows, -1).int()
    freq, spec = _rope(rot, interleaved)
    stride = heads * D

    def run(step):
        shape = ((rows * per_row + 2, hkv, page, D) if order == "head" else (rows * per_row + 2, page, hkv, D))
        both = [torch.full(shape, 0.5, dtype=TYPES[cache], device="cuda") for _ in range(2)]
        pools = [p if order == "head" else p.transpose(1, 2) for p in both]
        q_out = torch.full((n, hq, D), 9.0, dtype=qkv.dtype, device="cuda")
        cached = P.PagedCache(*pools)
        for i in range(0, n, step):
            part = qkv[i:i + step]
            P.aatc_paged_append(cached, table, len(part), part[:, hq:hq + hkv], part[:, hq + hkv:], stride,
                                stride, seq[i:], pos[i:], rope=spec, n_q_heads=hq, q=part[:, :hq],
                                q_tok_stride=stride, q_out=q_out[i:], q_out_tok_stride=hq * D)
        return pools, q_out
    (k, v), q_out = run(n)
    (k2, v2), q_out2 = run(n // 3 + 1)
    assert torch.equal(k, k2) and torch.equal(v, v2) and torch.equal(q_out, q_out2)
    assert torch.all(q_out[100:120] == 9.0)
    some = torch.tensor([0, 1, n // 2, n - 1], device="cuda")
    at = table[seq[some].long(), pos[some].long() // page].long()
    slot = pos[some].long() % page
    _close(q_out[some], *_turn(qkv[some][:, :hq], pos[some], freq, interleaved), qkv.dtype)
    _close(k[at, :, slot], *_turn(qkv[some][:, hq:hq + hkv], pos[some], freq, interleaved), k.dtype)
    assert torch.equal(v[at, :, slot], qkv[some][:, hq + hkv:].to(v.dtype))


@pytest.mark.parametrize("cache,qtype", [("f16", "f16"), ("f32", "f32"), ("bf16", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("lens", [[3000, 0, 17], [5000] + [40, 700] * 30, [33] * 600])
def test_attention_over_pools_past_the_caches(cache, qtype, lens):
    """Pools above 128 MiB: the bits of the same pages in smaller pools."""
    hq, hkv, page = 8, 4, 16
    g = torch.Generator(device="cuda").manual_seed(len(lens))
    per_row = -(-max(lens) // page)
    need = sum(-(-n // page) for n in lens)
    small = (torch.randn(2, need, hkv, page, D, generator=g, device="cuda") * 0.7).to(TYPES[cache])
    table = torch.full((len(lens), per_row), -1).int()
    at = 0
    for b, n in enumerate(lens):
        own = -(-n // page)
        table[b, :own] = torch.arange(at, at + own)
        at += own
    assert small.nbytes <= 128 << 20
    n_pages = (128 << 20) // (2 * hkv * page * D * small.element_size()) + need
    big = torch.full((2, n_pages, hkv, page, D), float("nan"), dtype=small.dtype, device="cuda")
    place = torch.randperm(n_pages, generator=g, device="cuda")[:need]
    big[:, place] = small
    moved = torch.where(table >= 0, place.cpu().int()[table.clamp(min=0).long()], table)
    q = torch.randn(len(lens), hq, D, generator=g, device="cuda").to(TYPES[qtype])
    n = torch.tensor(lens).int().cuda()
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(len(lens), hq, hkv), dtype=torch.uint8, device="cuda")
    outs = []
    for pools, t in ((small, table), (big, moved)):
        out, lse = torch.full((len(lens), hq, D), 5.0, device="cuda"), torch.empty(len(lens), hq, device="cuda")
        P.aatc_paged_decode_attention(P.PagedCache(pools[0], pools[1]), t.cuda(), n, len(lens), hq, q, D ** -0.5,
                                      out, ws, lse=lse)
        outs.append((out, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    k, v = (small[i].transpose(1, 2).reshape(-1, hkv, D) for i in (0, 1))
    for b in (0, len(lens) - 1):
        first = int(table[b, 0]) * page
        for j in (0, hq - 1):
            h = j // (hq // hkv)
            keys, values = (x[first:first + lens[b], h].double() for x in (k, v))
            want = torch.softmax(keys @ q[b, j].double() * D ** -0.5, 0) @ values
            assert (outs[1][0][b, j] - want).norm() <= 2e-6 * want.norm()


@pytest.mark.parametrize("page_bytes", [1 << 16, (1 << 16) + 16 * 5])
def test_copy_past_the_caches(page_bytes):
    """More than 512 MiB read and written: every page of some, and the pages left alone."""
    pairs_n = (512 << 20) // (2 * 4 * page_bytes) + 9
    n_pages = 2 * pairs_n + 3
    g = torch.Generator(device="cuda").manual_seed(5)
    pools = torch.randint(-2 ** 31, 2 ** 31 - 1, (4, n_pages, page_bytes // 4), generator=g, device="cuda",
                          dtype=torch.int32)
    order = torch.randperm(n_pages, generator=g, device="cuda")[:2 * pairs_n]
    pairs = order.reshape(pairs_n, 2).int().contiguous()
    pairs[3], pairs[7] = torch.tensor([-1, 2]).int(), torch.tensor([0, n_pages]).int()
    want = pools.clone()
    for i in range(0, pairs_n, 100):
        P.aatc_pages_copy(want, pairs[i:i + 100])
    good = pairs[(pairs[:, 0] >= 0) & (pairs[:, 1] < n_pages)].long()
    plain = pools.clone()
    plain[:, good[:, 1]] = pools[:, good[:, 0]]
    P.aatc_pages_copy(pools, pairs)
    assert torch.equal(pools, plain) and torch.equal(want, plain)
