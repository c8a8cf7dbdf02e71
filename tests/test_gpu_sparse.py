"""aatc_page_bounds and aatc_paged_sparse_attention against the 64-bit forms: bounds and picked pages
exactly, outputs within rounding."""
import math

import pytest
import torch

import paper_2608_14191_amd as P
from drafts_ref import page_bounds, sparse_attention
from paged_ref import TYPES, pool, to_cuda

pytestmark = pytest.mark.gpu
D = 128
SCALE = D ** -0.5
NAN = float("nan")


def _case(seed, lens, hq, hkv, page, cache="bf16", qtype="bf16", order="head", holes=(), keys=None):
    """Pools, table (pages in random order, garbage behind the sequences), lengths, queries, and the
    bounds of all pages that the sequences have."""
    g = torch.Generator().manual_seed(seed)
    batch, per_row = len(lens), max(1, -(-max(lens) // page))
    n_pages = batch * per_row + 2
    k = pool(g, n_pages, hkv, page, TYPES[cache], order)
    v = pool(g, n_pages, hkv, page, TYPES[cache], order)
    # (pages that differ: a share of each page's keys is its own)
    k += torch.randn(n_pages, hkv, 1, D, generator=g).to(k.dtype)
    if keys:
        keys(k)
    table = torch.randperm(n_pages, generator=g)[:batch * per_row].reshape(-1, per_row).int()
    codes = torch.full((n_pages, hkv, 2, D), 99, dtype=torch.int8)
    scales = torch.full((n_pages, hkv), NAN)
    for b, n in enumerate(lens):
        for i in range(per_row):
            lo, at = min(max(n - i * page, 0), page), int(table[b, i])
            k[at, :, lo:], v[at, :, lo:] = NAN, math.inf
            for h in range(hkv):
                if lo:
                    codes[at, h], scales[at, h] = page_bounds(k[at, h, :lo])
    for b, i, entry in holes:
        table[b, i] = entry
    q = torch.randn(batch, hq, D, generator=g).to(TYPES[qtype])
    return dict(k=k, v=v, table=table, lens=torch.tensor(lens).int(), q=q, codes=codes, scales=scales)


def _bounds(c, held, wanted, codes=None, scales=None):
    codes = torch.full(c["codes"].shape, 99, dtype=torch.int8) if codes is None else codes
    scales = torch.full(c["scales"].shape, NAN) if scales is None else scales
    codes, scales = codes.cuda(), scales.cuda()
    P.aatc_page_bounds(P.PagedCache(to_cuda(c["k"]), to_cuda(c["v"])), c["table"].cuda(),
                       None if held is None else torch.tensor(held).int().cuda(),
                       torch.tensor(wanted).int().cuda(), codes, scales)
    torch.cuda.synchronize()
    return codes.cpu(), scales.cpu()


def _same(x, y):
    return torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("cache", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("page", [8, 16, 64, 512])
def test_bounds_of_whole_sequences(cache, order, page):
    lens = [0, 1, 7, 8, 9, 100, 513]
    c = _case(1, lens, 3, 3, page, cache, order=order)
    codes, scales = _bounds(c, None, lens)
    assert _same(codes, c["codes"]) and _same(scales, c["scales"])


def test_bounds_of_new_tokens():
    """Only the pages of new tokens, of all their tokens; lengths are clamped; holes are skipped."""
    lens = [100, 37, 64, 20, 16, 0, 90]
    c = _case(2, lens, 2, 2, 16, holes=[(6, 2, -1), (6, 3, 10 ** 6)])
    held = [90, 37, 48, 17, 16, 0, -5]
    codes, scales = _bounds(c, held, lens)
    for b, (a, z) in enumerate(zip(held, lens)):
        for i in range(c["table"].shape[1]):
            at = int(c["table"][b, i])
            if not 0 <= at < c["codes"].shape[0]:
                continue
            new = max(a, 0) < min((i + 1) * 16, z) and z > i * 16 and z > a
            want = (c["codes"][at], c["scales"][at]) if new else \
                (torch.full_like(codes[at], 99), torch.full_like(scales[at], NAN))
            assert _same(codes[at], want[0]) and _same(scales[at], want[1]), (b, i)
    wide = [10 ** 6, 37, 64, 20, 16, 0, 90]         # clamped to the table's 112 tokens: garbage within
    codes, scales = _bounds(c, [96] + lens[1:], wide)
    at = int(c["table"][0, 6])
    assert torch.all(scales[at] == math.inf) and torch.all(codes[at] == 0)


@pytest.mark.parametrize("cache", ["bf16", "f16", "f32"])
def test_bounds_of_odd_values(cache):
    """Zeros, powers of two, values that 127 steps just reach, the smallest and largest, no number."""
    top = torch.finfo(TYPES[cache]).max
    tiny = torch.finfo(TYPES[cache]).smallest_normal

    def keys(k):
        k[0] = 0
        k[1] = 1.0
        k[2] = -127 / 128
        k[3, :, 0], k[3, :, 1:] = 127.5 / 128, 0.25
        k[4] = tiny
        k[5, :, 0], k[5, :, 1:] = 1.0, -tiny
        k[6, :, 0, 0] = top
        k[7, :, 2, 5] = NAN
        k[8, :, 2, 5] = -math.inf
        k[9, :, :, ::2] = 2.0 ** -14
        k[10, :, 0, 1], k[10, :, 1:, 2] = 3.0, -1e-5
    lens = [16 * 14]
    c = _case(3, lens, 2, 2, 16, cache, keys=keys)
    codes, scales = _bounds(c, None, lens)
    assert _same(codes, c["codes"]) and _same(scales, c["scales"])
    at = torch.isfinite(scales).nonzero(as_tuple=True)
    real = codes[at].double() * scales[at].double()[:, None, None]
    for p, h, r in zip(*at, real):
        if torch.isfinite(c["k"][p, h]).all():
            assert torch.all(r[0] >= c["k"][p, h].double().amax(0)) and torch.all(r[1] <= c["k"][p, h].double().amin(0))


@pytest.mark.parametrize("rows", [1, 255, 256, 257, 1500])
def test_bounds_of_many_rows(rows):
    lens = [(13 * b) % 40 for b in range(rows)]
    lens[rows // 2] = 700
    c = _case(4, lens, 1, 1, 8)
    codes, scales = _bounds(c, None, lens)
    assert _same(codes, c["codes"]) and _same(scales, c["scales"])


def _run(c, most, first=1, last=1, lse=True, workspace=None, **more):
    batch, hq, _ = c["q"].shape
    hkv = c["k"].shape[1]
    out = torch.full((batch, hq, D), NAN, device="cuda")
    out_lse = torch.full((batch, hq), NAN, device="cuda")
    picked = torch.full((batch, hkv, most), 99, dtype=torch.int32, device="cuda")
    if workspace is None:
        workspace = torch.zeros(P.aatc_paged_sparse_workspace_bytes(batch, hq, hkv, c["table"].shape[1]),
                                dtype=torch.uint8, device="cuda")
    P.aatc_paged_sparse_attention(P.PagedCache(to_cuda(c["k"]), to_cuda(c["v"])), c["table"].cuda(),
                                  c["lens"].cuda(), c["codes"].cuda(), c["scales"].cuda(), batch, hq,
                                  c["q"].cuda(), more.pop("scale", SCALE), picked, out, workspace,
                                  first=first, last=last, lse=out_lse if lse else None, **more)
    torch.cuda.synchronize()
    return picked.cpu(), out.cpu(), out_lse.cpu()


def _check(c, most, first=1, last=1, **more):
    picked, got, lse = _run(c, most, first, last, **more)
    want_picked, want, want_lse, spread = sparse_attention(
        c["k"], c["v"], c["codes"], c["scales"], c["table"], c["lens"], c["q"], more.get("scale", SCALE),
        most, first, last, more.get("softcap", 0.0))
    for b, row in enumerate(want_picked):
        for h, some in enumerate(row):
            assert picked[b, h].tolist() == some + [-1] * (most - len(some)), (b, h)
    # Rounding: as in the attention over whole sequences (a key's square is twice as large here: 2^-24
    # of 128 products below 23 * 1.5 each), relative to sum p |v|.
    eps = 128 * 2.0 ** -24 * 35 + 2.0 ** -17
    assert torch.all((got.double() - want).abs() <= eps * spread + 1e-30)
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), empty)
    assert torch.all((lse.double() - want_lse)[~empty].abs() <= eps * (1 + want_lse[~empty].abs()))
    assert torch.all(got[empty] == 0)
    norm = want.norm()
    assert norm == 0 or (got.double() - want).norm() <= 2e-6 * norm
    return picked, got


@pytest.mark.parametrize("cache,qtype", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "f32"),
                                         ("f16", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("order", ["head", "token"])
def test_types_and_orders(cache, qtype, order):
    _check(_case(10, [300, 0, 1, 77, 160], 8, 2, 16, cache, qtype, order), 6)


@pytest.mark.parametrize("page", [8, 16, 32, 128])
@pytest.mark.parametrize("most", [1, 2, 3, 8, 17, 64])
def test_pages_and_counts(page, most):
    _check(_case(11, [1000, 33, 8, 511], 4, 2, page), most, first=0 if most == 1 else 1)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (7, 1), (28, 4), (20, 1), (33, 3), (64, 2), (256, 1)])
@pytest.mark.parametrize("cache", ["bf16", "f32"])
def test_heads(hq, hkv, cache):
    _check(_case(12, [400, 90], hq, hkv, 16, cache, cache), 5)


@pytest.mark.parametrize("first,last", [(0, 0), (0, 1), (1, 0), (3, 2), (0, 6), (6, 0)])
def test_pages_that_are_picked_always(first, last):
    _check(_case(13, [300, 50, 16, 113], 4, 2, 16), 6, first, last)


@pytest.mark.parametrize("cap", [5.0, 1e29, 2e30])
@pytest.mark.parametrize("scale", [SCALE, -SCALE, 0.0])
def test_caps_and_scales(cap, scale):
    _check(_case(14, [300, 50], 4, 2, 16), 5, softcap=cap, scale=scale)


def test_pages_that_are_not_there():
    holes = [(0, 0, -1), (0, 7, 10 ** 6), (1, 3, -1), (2, 0, -1), (2, 1, -1), (2, 2, -7)]
    c = _case(15, [300, 64, 48], 4, 2, 16, holes=holes)
    _, got = _check(c, 5)
    assert torch.all(got[2] == 0)
    _check(c, 40)


def test_equal_scores():
    """Pages of the same keys: the lowest indexes."""
    def keys(k):
        k[:] = k[:1]
    _check(_case(16, [500, 64], 4, 2, 8, keys=keys), 9)
    c = _case(16, [500, 64], 4, 2, 8)
    c["q"][:] = 0                                  # every score is 0
    _check(c, 9)


def test_keys_and_queries_that_are_not_finite():
    """Pages without finite bounds come first; heads that are not finite have no say, and get NaN."""
    c = _case(17, [320, 320], 4, 2, 16)
    for b, i in ((0, 5), (0, 9), (1, 11)):
        at = int(c["table"][b, i])
        c["k"][at, 0, 3, 7] = -math.inf
        c["codes"][at, 0], c["scales"][at, 0] = page_bounds(c["k"][at, 0])
    c["q"][:, 0, 7] = 1.0
    c["q"][:, 1, 7] = 2.0                          # their scores are -infinity: no weight
    _check(c, 6)
    c["q"][0, 0, 3], c["q"][1, 2, 3], c["q"][1, 3, 3] = NAN, math.inf, -math.inf
    clean = dict(c, q=c["q"].clone())
    picked, got, lse = _run(c, 6)
    want = sparse_attention(c["k"], c["v"], c["codes"], c["scales"], c["table"], c["lens"], c["q"], SCALE,
                            6, 1, 1)[0]
    assert picked.tolist() == [[x + [-1] * (6 - len(x)) for x in row] for row in want]
    assert torch.isnan(got[0, 0]).all() and torch.isfinite(got[0, 1:]).all()
    assert torch.isfinite(got[1, :2]).all() and torch.equal(clean["q"].isnan(), c["q"].isnan())


def test_scales_that_were_never_set():
    """Any bits in some pages' bounds: as many pages as there is room for, in order, and no more."""
    for bits in (0x7fffffff, -1, 0x7fc00000, -4194304, 0x7f800001):
        c = _case(25, [320, 250], 4, 2, 16)
        wild = torch.full(c["scales"].shape, bits, dtype=torch.int32).view(torch.float32)
        c["scales"][::2] = wild[::2]
        c["codes"][::3] = -128
        picked, got, lse = _run(c, 6)
        for b, pages in ((0, 20), (1, 16)):
            for h in range(2):
                x = picked[b, h].tolist()
                assert x == sorted(set(x)) and x[0] == 0 and x[-1] == pages - 1
        assert torch.isfinite(got).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("n,most", [(60000, 100), (200000, 300), (200000, 8200)])
def test_many_pages(n, most):
    """More pages than a workgroup has in registers, more picked than it lists; parts joined."""
    c = _case(18, [n, 70], 2, 1, 8, "f16", "f16")
    _check(c, most, first=2, last=3)


@pytest.mark.parametrize("batch,hkv", [(33, 8), (300, 1)])
def test_many_rows(batch, hkv):
    lens = [(37 * b) % 400 for b in range(batch)]
    lens[batch // 2] = 2000
    _check(_case(19, lens, 2 * hkv, hkv, 16), 7)


def test_picked_pages_match_all_pages():
    """With room for all pages it is aatc_paged_decode_attention."""
    c = _case(20, [500, 31], 8, 2, 16)
    _, got = _check(c, 64)
    cache = P.PagedCache(to_cuda(c["k"]), to_cuda(c["v"]))
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(2, 8, 2), dtype=torch.uint8, device="cuda")
    out = torch.empty(2, 8, D, device="cuda")
    P.aatc_paged_decode_attention(cache, c["table"].cuda(), c["lens"].cuda(), 2, 8, c["q"].cuda(), SCALE,
                                  out, ws)
    assert (out.cpu() - got).norm() <= 2e-6 * got.norm()


def test_a_workspace_for_calls_of_all_shapes():
    cases = [(_case(21, [4000], 4, 1, 16), 100), (_case(22, [300] * 8, 16, 8, 16), 5),
             (_case(23, [9000, 100], 20, 1, 8), 500)]
    most_bytes = max(P.aatc_paged_sparse_workspace_bytes(*c["q"].shape[:2], c["k"].shape[1], c["table"].shape[1])
                     for c, _ in cases)
    ws = torch.zeros(most_bytes, dtype=torch.uint8, device="cuda")
    for turn in range(2):
        for c, most in cases:
            x, y = _run(c, most, workspace=ws), _run(c, most, workspace=ws)
            assert all(torch.equal(i, j) for i, j in zip(x, y))
            if turn == 0:
                _check(c, most, workspace=ws)


def test_steps_of_a_sequence_in_a_graph():
    """Append, bounds of the new token's page, attention: captured and replayed as the sequence grows."""
    hq, hkv, page, per_row = 4, 2, 8, 20
    g = torch.Generator().manual_seed(24)
    k, v = (torch.zeros(per_row, hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = P.PagedCache(k, v)
    table = torch.randperm(per_row, generator=g).int()[None].cuda()
    codes = torch.zeros(per_row, hkv, 2, D, dtype=torch.int8, device="cuda")
    scales = torch.zeros(per_row, hkv, device="cuda")
    held, wanted = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (0, 1))
    new = torch.zeros(1, hq + 2 * hkv, D, dtype=torch.bfloat16, device="cuda")
    stride = (hq + 2 * hkv) * D
    ws = torch.zeros(P.aatc_paged_sparse_workspace_bytes(1, hq, hkv, per_row), dtype=torch.uint8, device="cuda")
    out = torch.zeros(1, hq, D, device="cuda")
    picked = torch.zeros(1, hkv, 4, dtype=torch.int32, device="cuda")

    def step():
        P.aatc_paged_append(cache, table, 1, new[:, hq:hq + hkv], new[:, hq + hkv:], stride, stride, None, held)
        P.aatc_page_bounds(cache, table, held, wanted, codes, scales)
        P.aatc_paged_sparse_attention(cache, table, wanted, codes, scales, 1, hq, new[:, :hq], SCALE, picked,
                                      out, ws, first=1, last=1)
        held.add_(1)
        wanted.add_(1)
    graph = None
    for t in range(150):
        x = torch.randn(1, hq + 2 * hkv, D, generator=g).bfloat16()
        new.copy_(x)
        if t == 3:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        graph.replay() if graph else step()
        if t in (0, 2, 7, 8, 40, 41, 100, 149):
            torch.cuda.synchronize()
            c = [y.cpu() for y in (k, v, codes, scales, table)]
            want_picked, want, _, _ = sparse_attention(*c, torch.tensor([t + 1]), x[:, :hq], SCALE, 4, 1, 1)
            for i in range(t // page + 1):
                for h in range(hkv):
                    lo = min(page, t + 1 - i * page)
                    b = page_bounds(c[0][int(c[4][0, i]), h, :lo])
                    assert _same(c[2][int(c[4][0, i]), h], b[0]) and float(c[3][int(c[4][0, i]), h]) == b[1]
            assert picked.cpu().tolist() == [[p + [-1] * (4 - len(p)) for p in want_picked[0]]]
            assert (out.cpu().double() - want).norm() <= 2e-6 * want.norm()
