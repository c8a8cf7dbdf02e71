"""aatc_paged_decode_attention against the 64-bit form: types, page sizes and orders, lengths from
nothing on, windows, sinks, caps, biases, pages that are not there, rows that nothing is left of."""
import math

import pytest
import torch

import paper_2608_14191_amd as P
from paged_ref import HALF_STEP, TYPES, attention, pool, to_cuda

pytestmark = pytest.mark.gpu
D = 128
NAN = float("nan")


def _case(seed, lens, hq, hkv, page, cache="bf16", qtype="bf16", order="head", holes=()):
    """Pools, table (pages in random order, garbage behind the sequences), lengths, queries."""
    g = torch.Generator().manual_seed(seed)
    per_row = max(1, -(-max(lens) // page)) + 1
    n_pages = len(lens) * per_row + 2
    k = pool(g, n_pages, hkv, page, TYPES[cache], order)
    v = pool(g, n_pages, hkv, page, TYPES[cache], order)
    table = torch.randperm(n_pages, generator=g)[:len(lens) * per_row].reshape(-1, per_row).int()
    for b, n in enumerate(lens):
        for i in range(per_row):
            lo = min(max(n - i * page, 0), page)
            k[table[b, i].long(), :, lo:] = NAN
            v[table[b, i].long(), :, lo:] = math.inf
    for b, i, entry in holes:
        table[b, i] = entry
    q = torch.randn(len(lens), hq, D, generator=g).to(TYPES[qtype])
    return k, v, table, torch.tensor(lens, dtype=torch.int32), q


def _run(k, v, table, lens, q, lse=True, workspace=None, **more):
    batch, hq, hkv = q.shape[0], q.shape[1], k.shape[1]
    cache = P.PagedCache(to_cuda(k), to_cuda(v))
    out = torch.full((batch, hq, D), NAN, device="cuda")
    out_lse = torch.full((batch, hq), NAN, device="cuda")
    if workspace is None:
        workspace = torch.zeros(P.aatc_paged_decode_workspace_bytes(batch, hq, hkv),
                                dtype=torch.uint8, device="cuda")
    slopes = more.pop("slopes", None)
    P.aatc_paged_decode_attention(cache, table.cuda(), lens.cuda(), batch, hq, q.cuda(), D ** -0.5,
                                  out, workspace, lse=out_lse if lse else None,
                                  slopes=None if slopes is None else slopes.cuda(), **more)
    torch.cuda.synchronize()
    return out.cpu(), out_lse.cpu()


def _check(case, **more):
    k, v, table, lens, q = case
    got, lse = _run(*case, **more)
    more = dict(more)
    want, want_lse, spread = attention(k, v, table, lens, q, D ** -0.5, more.get("window", 0),
                                       more.get("sink", 0), more.get("softcap", 0.0),
                                       more.get("slopes"))
    # Rounding: a score is a sum of 128 products in fp32 in some order, off by at most
    # 128 2^-24 sum |q k| scale, and its weight by as much, relative (|q|, |k| near sqrt(128):
    # sum |q k| scale < 11.4 * 2 for these draws); cap and bias add a few ulps of |z| < 2^6;
    # weights and sums some 2^-22 more.  All of it relative to sum p |v|.
    eps = 128 * 2.0 ** -24 * 23 + 2.0 ** -17
    assert torch.all((got.double() - want).abs() <= eps * spread + 1e-30)
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), empty)
    assert torch.all((lse.double() - want_lse)[~empty].abs() <= eps * (1 + want_lse[~empty].abs()))
    assert torch.all(got[empty] == 0)
    # and on the whole much closer than that bound
    norm = want.norm()
    assert norm == 0 or (got.double() - want).norm() <= 2e-6 * norm
    return got


@pytest.mark.parametrize("cache,qtype", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"),
                                         ("bf16", "f32"), ("f16", "f32"), ("f16", "bf16"),
                                         ("bf16", "f16"), ("f32", "bf16")])
@pytest.mark.parametrize("order", ["head", "token"])
def test_types_and_orders(cache, qtype, order):
    _check(_case(1, [77, 0, 1, 300], 8, 2, 16, cache, qtype, order))


@pytest.mark.parametrize("page", [8, 16, 32, 64, 256])
@pytest.mark.parametrize("cache", ["bf16", "f32"])
def test_page_sizes(page, cache):
    _check(_case(2, [1, 7, 8, 9, 31, 32, 33, 64, 129, 500], 4, 4, page, cache))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (7, 1), (16, 1), (17, 1), (40, 2), (28, 4), (64, 8)])
def test_head_groups(hq, hkv):
    _check(_case(3, [130, 45], hq, hkv, 16))


@pytest.mark.parametrize("cache", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 4), (20, 4), (33, 33), (64, 0), (100, 1),
                                         (300, 10), (5000, 4), (16, 2000)])
def test_windows_and_sinks(cache, window, sink):
    _check(_case(4, [1, 19, 20, 500, 64, 333, 0, 1030], 4, 2, 16, cache), window=window, sink=sink)


@pytest.mark.parametrize("cache", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cap,biased", [(5.0, False), (50.0, True), (0.0, True), (0.3, True)])
def test_caps_and_biases(cache, cap, biased):
    slopes = torch.logspace(-1, -8, 8, base=2.0) if biased else None
    _check(_case(5, [200, 3, 97], 8, 2, 32, cache), softcap=cap, slopes=slopes)


def test_pages_that_are_not_there():
    """Negative, too large and far entries: their tokens are not attended, nothing is read there;
    a row without any page gets zeros."""
    holes = [(0, 1, -1), (0, 3, 10 ** 6), (1, 0, -2 ** 31), (2, 0, -1), (2, 1, -1), (3, 2, 2 ** 31 - 1)]
    got = _check(_case(6, [70, 40, 20, 90], 4, 2, 16, holes=holes))
    assert torch.all(got[2] == 0)


def test_lengths_out_of_range_are_clamped():
    k, v, table, lens, q = _case(7, [64, 33], 4, 2, 16)
    table = table[:, :4].contiguous()
    k, v = torch.nan_to_num(k, nan=0.5), torch.nan_to_num(v, posinf=0.25)
    got, _ = _run(k, v, table, torch.tensor([10 ** 9, -5], dtype=torch.int32), q)
    want, _, _ = attention(k, v, table, [64, 0], q, D ** -0.5)
    assert (got.double() - want).norm() <= 2e-6 * want.norm()
    assert torch.all(got[1] == 0)


@pytest.mark.parametrize("lens", [[3000], [9000, 1, 0, 700], [257] * 40, [33] * 700, [5000, 5001]])
@pytest.mark.parametrize("cache", ["bf16", "f32"])
def test_splits(lens, cache):
    """Rows of many workgroups, of a part of one, and many rows to a workgroup."""
    _check(_case(8, lens, 4, 2, 16, cache))


@pytest.mark.parametrize("hq,hkv,lens", [
    (16, 1, [9000]), (40, 2, [6000, 3, 4100]), (1, 1, [20000]),           # runs, many heads to join
    (1, 1, [40 * i for i in range(128)]), (2, 1, [7] * 65 + [6000] + [0] * 62),   # 128 rows
    (64, 4, [5] * 33 + [8000]), (16, 1, [0] * 150 + [5000, 9000]),        # lines, a row in many
    (7, 1, [600] * 129), (4, 4, [1100, 20] * 30)])
def test_splits_of_rows(hq, hkv, lens):
    _check(_case(12, lens, hq, hkv, 64))


def test_peaked_scores_and_far_maximum():
    """Queries along one key (a weight near 1), and scores far below the maximum."""
    k, v, table, lens, q = _case(9, [900, 1200], 4, 2, 16, "f16", "f32")
    for b, t in ((0, 5), (1, 1199)):
        page, slot = int(table[b, t // 16]), t % 16
        for j in range(4):
            q[b, j] = k[page, j // 2, slot].float() * 8
    _check((k, v, table, lens, q))


def test_query_stride_and_workspace_reuse():
    k, v, table, lens, q = _case(10, [700, 64, 1], 8, 2, 16)
    wide = torch.randn(3, 1000 + 8 * D).to(torch.bfloat16)
    wide[:, :8 * D] = q.reshape(3, -1)
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(3, 8, 2), dtype=torch.uint8, device="cuda")
    a, _ = _run(k, v, table, lens, q, workspace=ws)
    cache = P.PagedCache(to_cuda(k), to_cuda(v))
    out = torch.empty(3, 8, D, device="cuda")
    for _ in range(3):
        out.fill_(NAN)
        P.aatc_paged_decode_attention(cache, table.cuda(), lens.cuda(), 3, 8, wide.cuda(),
                                      D ** -0.5, out, ws, q_stride=1000 + 8 * D)
        assert torch.equal(out.cpu(), a)
    # a smaller call on the same workspace
    b, _ = _run(k, v, table[1:], lens[1:], q[1:], workspace=ws)
    want, _, _ = attention(k, v, table[1:], lens[1:], q[1:], D ** -0.5)
    assert (b.double() - want).norm() <= 2e-6 * want.norm()


def test_workspace_of_calls_of_other_shapes():
    """One workspace, large enough for all: few rows and many, few heads and many, in turn."""
    cases = [_case(20, [900] * 3, 16, 1, 16), _case(21, [40, 300, 90] * 50, 2, 1, 16),
             _case(22, [5000], 32, 8, 16), _case(23, [20, 2600] * 12, 12, 12, 16)]
    ws = torch.zeros(max(P.aatc_paged_decode_workspace_bytes(c[4].shape[0], c[4].shape[1], c[0].shape[1])
                         for c in cases), dtype=torch.uint8, device="cuda")
    want = [_run(*c)[0] for c in cases]
    for i in (0, 1, 2, 3, 1, 0, 3, 2, 1):
        assert torch.equal(_run(*cases[i], workspace=ws)[0], want[i]), i


def test_non_finite_queries_and_values():
    k, v, table, lens, q = _case(11, [50, 50], 4, 2, 16)
    q[0, 1, 3] = NAN
    v[int(table[1, 0]), 0, 2, 7] = math.inf
    got, _ = _run(k, v, table, lens, q)
    assert torch.all(torch.isnan(got[0, 1]))
    assert torch.all(torch.isfinite(got[0, [0, 2, 3]]))
    assert not torch.any(torch.isfinite(got[1, :2, 7]))
    assert torch.all(torch.isfinite(got[1, :2, :7])) and torch.all(torch.isfinite(got[1, 2:]))


@pytest.mark.parametrize("cache,qtype", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "f32"),
                                         ("f16", "bf16")])
def test_queries_of_any_alignment(cache, qtype):
    """Sequences an odd number of elements apart, the first behind an odd offset."""
    k, v, table, lens, q = _case(30, [100, 3, 260], 4, 2, 16, cache, qtype)
    want, _ = _run(k, v, table, lens, q)
    stride = 4 * D + 3
    flat = torch.zeros(1 + 3 * stride, dtype=q.dtype)
    flat[1:].reshape(3, stride)[:, :4 * D] = q.reshape(3, -1)
    out = torch.empty(3, 4, D, device="cuda")
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(3, 4, 2), dtype=torch.uint8, device="cuda")
    P.aatc_paged_decode_attention(P.PagedCache(to_cuda(k), to_cuda(v)), table.cuda(), lens.cuda(), 3, 4,
                                  flat.cuda()[1:], D ** -0.5, out, ws, q_stride=stride)
    assert torch.equal(out.cpu(), want)


def test_two_calls_at_once():
    """Two streams, a workspace each: the results of one after the other."""
    cases = [_case(31, [3000, 5], 8, 2, 16), _case(32, [50, 900] * 40, 8, 4, 16)]
    want = [_run(*c)[0] for c in cases]
    held, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k, v, table, lens, q in cases:
        ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(len(lens), q.shape[1], k.shape[1]),
                         dtype=torch.uint8, device="cuda")
        held.append((P.PagedCache(to_cuda(k), to_cuda(v)), table.cuda(), lens.cuda(), q.cuda(),
                     torch.zeros(*q.shape, device="cuda"), ws))
    torch.cuda.synchronize()
    for _ in range(20):
        for (cache, table, lens, q, out, ws), stream in zip(held, streams):
            P.aatc_paged_decode_attention(cache, table, lens, len(lens), q.shape[1], q, D ** -0.5, out,
                                          ws, stream=stream.cuda_stream)
    torch.cuda.synchronize()
    for (*_, out, _), w in zip(held, want):
        assert torch.equal(out.cpu(), w)


@pytest.mark.parametrize("order", ["head", "token"])
def test_pools_past_32_bit_offsets(order):
    """Pages at the end of pools of 2^31 elements and more: append, attention and copy reach them."""
    hkv, page, n = 8, 64, 150
    n_pages = (1 << 31) // (hkv * page * D) + 5
    shape = (n_pages, hkv, page, D) if order == "head" else (n_pages, page, hkv, D)
    both = torch.zeros((2, *shape), dtype=torch.bfloat16, device="cuda")
    pools = [x if order == "head" else x.transpose(1, 2) for x in both]
    cache = P.PagedCache(*pools)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 3]], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(1)
    x = torch.randn(n, 2 * hkv, D, generator=g).to(torch.bfloat16)
    dev = x.cuda()
    P.aatc_paged_append(cache, table, n, dev[:, :hkv], dev[:, hkv:], 2 * hkv * D, 2 * hkv * D,
                        torch.zeros(n, dtype=torch.int32, device="cuda"),
                        torch.arange(n, dtype=torch.int32, device="cuda"))
    P.aatc_pages_copy(both, torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda"))
    table[0, 0] = n_pages - 2
    both[:, n_pages - 1] = NAN
    q = torch.randn(1, hkv, D, generator=g)
    out = torch.empty(1, hkv, D, device="cuda")
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(1, hkv, hkv), dtype=torch.uint8, device="cuda")
    P.aatc_paged_decode_attention(cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), 1,
                                  hkv, q.cuda(), D ** -0.5, out, ws)
    got = out.cpu().double()
    for h in range(hkv):
        k, v = x[:, h].double(), x[:, hkv + h].double()
        want = torch.softmax(k @ q[0, h].double() * D ** -0.5, 0) @ v
        assert (got[0, h] - want).norm() <= 2e-6 * want.norm()


def test_what_the_binding_refuses():
    """(A slice of a longer tensor of queries is not refused: what is read lies in its storage.)"""
    k, v, table, lens, q = _case(33, [20, 30], 4, 2, 16)
    cache = P.PagedCache(k.cuda(), v.cuda())
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(2, 4, 2), dtype=torch.uint8, device="cuda")
    good = dict(cache=cache, table=table.cuda(), seq_len=lens.cuda(), batch=2, n_q_heads=4, q=q.cuda(),
                softmax_scale=0.1, out=torch.empty(2, 4, D, device="cuda"), workspace=ws)
    P.aatc_paged_decode_attention(**good)
    bad = [dict(q=q), dict(table=table), dict(seq_len=lens), dict(out=torch.empty(2, 4, D)),
           dict(out=torch.empty(1, 4, D, device="cuda")), dict(out=good["out"].bfloat16()),
           dict(seq_len=lens.cuda().long()), dict(seq_len=lens.cuda()[:1]), dict(q=q[:1].cuda()),
           dict(table=table.cuda().long()), dict(table=table.cuda().T), dict(batch=3),
           dict(workspace=ws[:256]), dict(workspace=ws.cpu()), dict(slopes=torch.ones(3, device="cuda")),
           dict(lse=torch.ones(7, device="cuda")), dict(q=q.cuda().transpose(1, 2).contiguous().transpose(1, 2))]
    for change in bad:
        with pytest.raises(P.AatcError):
            P.aatc_paged_decode_attention(**{**good, **change})
    with pytest.raises(TypeError):
        P.aatc_paged_decode_attention(**{**good, "q": q.cuda().double()})
    for a, b in ((k.cuda(), v), (k, v)):
        with pytest.raises(P.AatcError):
            P.PagedCache(a, b)
    for a, b in ((k.cuda(), v.cuda()[:3]), (k.cuda(), v.cuda().float()), (k.cuda()[0], v.cuda()[0]),
                 (k.cuda().transpose(2, 3).contiguous().transpose(2, 3), v.cuda())):
        with pytest.raises(ValueError):
            P.PagedCache(a, b)
    torch.cuda.synchronize()
