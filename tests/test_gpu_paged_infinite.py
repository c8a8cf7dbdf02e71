"""Infinite scores in the attention over pages, alone and joined with a compressed cache: a head all
of whose attended scores are -infinity has the NaN of its softmax, not the zeros of one without
tokens; other infinite scores follow the formula."""
import math

import pytest
import torch

import paper_2608_14191_amd as P
from helpers import alpha_cache, device_params, record_cache, tile_cache
from kvsynth import workload
from oracle import aatc as ora
from paged_ref import TYPES, attention, pool, to_cuda

pytestmark = pytest.mark.gpu
D = 128
NAN = float("nan")
CHANNEL = 37


def _case(seed, lens, hq, hkv, cache, qtype, page=16):
    g = torch.Generator().manual_seed(seed)
    per_row = max(1, -(-max(lens) // page))
    n_pages = len(lens) * per_row + 1
    k, v = (pool(g, n_pages, hkv, page, TYPES[cache]) for _ in range(2))
    table = torch.randperm(n_pages, generator=g)[:len(lens) * per_row].reshape(-1, per_row).int()
    q = torch.randn(len(lens), hq, D, generator=g).to(TYPES[qtype])
    return k, v, table, torch.tensor(lens).int(), q


def _run(k, v, table, lens, q, **more):
    batch, hq, hkv = q.shape[0], q.shape[1], k.shape[1]
    out = torch.full((batch, hq, D), 5.0, device="cuda")
    lse = torch.full((batch, hq), 5.0, device="cuda")
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(batch, hq, hkv), dtype=torch.uint8, device="cuda")
    P.aatc_paged_decode_attention(P.PagedCache(to_cuda(k), to_cuda(v)), table.cuda(), lens.cuda(), batch,
                                  hq, q.cuda(), D ** -0.5, out, ws, lse=lse, **more)
    return out.cpu(), lse.cpu()


def _finite_alike(got, want):
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = torch.isfinite(want)
    # (2e-6: 2^-19, below the sum of 128 products' roundings, 128 2^-24, times scores near 1)
    assert (got.double() - want)[ok].norm() <= 2e-6 * want[ok].norm()


# Rows in runs (few), waves with whole rows, waves and workgroups with shares of rows.
SHAPES = [([1], 1, 1), ([300, 0, 5], 4, 2), ([9000, 64], 4, 2), ([20000], 2, 1), ([33] * 700, 2, 1),
          ([40, 300, 0, 90] * 40, 2, 1), ([5] * 33 + [3000, 0], 32, 4), ([600] * 129, 1, 1)]


@pytest.mark.parametrize("cache,qtype", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("lens,hq,hkv", SHAPES)
def test_every_score_minus_infinity(cache, qtype, lens, hq, hkv):
    """An infinite query channel, of opposite sign in every key: NaN; rows of no token: zeros."""
    k, v, table, n, q = _case(1, lens, hq, hkv, cache, qtype)
    k[..., CHANNEL] = -k[..., CHANNEL].abs() - 0.125
    q[::2, 0, CHANNEL] = math.inf
    got, lse = _run(k, v, table, n, q)
    want, want_lse, _ = attention(k, v, table, n.tolist(), q, D ** -0.5)
    hit = torch.zeros(len(lens), hq, dtype=torch.bool)
    hit[::2, 0] = n[::2] > 0
    assert torch.all(torch.isnan(got[hit])) and torch.all(torch.isnan(want[hit]))
    assert torch.all(lse[hit] == -math.inf) and torch.all(want_lse[hit] == -math.inf)
    assert torch.all(got[n == 0] == 0) and torch.all(lse[n == 0] == -math.inf)
    _finite_alike(got, want)


@pytest.mark.parametrize("lens,window,sink", [([500, 1, 0, 64], 1, 0), ([500, 3, 700], 20, 4)])
def test_every_attended_score_minus_infinity(lens, window, sink):
    """Only attended tokens count, and only those make a head one that has tokens; holes do not."""
    k, v, table, n, q = _case(2, lens, 4, 2, "bf16", "bf16")
    q[:, 1, CHANNEL] = math.inf
    for b, m in enumerate(lens):
        for t in range(m):
            if t >= m - window or t < sink:
                at = int(table[b, t // 16])
                k[at, :, t % 16, CHANNEL] = -k[at, :, t % 16, CHANNEL].abs() - 0.125
    table[0] = -1                                        # a row whose pages are not there
    got, lse = _run(k, v, table, n, q, window=window, sink=sink)
    want, _, _ = attention(k, v, table, lens, q, D ** -0.5, window, sink)
    empty = torch.tensor([b == 0 or m == 0 for b, m in enumerate(lens)])
    assert torch.all(got[empty] == 0) and torch.all(lse[empty] == -math.inf)
    assert torch.all(torch.isnan(got[~empty, 1]))
    _finite_alike(got, want)


def test_scores_that_overflow_downwards():
    """Finite queries and keys whose products pass float32's range."""
    k, v, table, n, q = _case(3, [200, 3000], 4, 2, "f32", "f32")
    k[..., CHANNEL] = k[..., CHANNEL].abs() + 2.0
    q[0, 2, CHANNEL] = q[1, 0, CHANNEL] = -3e38
    got, lse = _run(k, v, table, n, q)
    assert torch.all(torch.isnan(got[0, 2])) and torch.all(torch.isnan(got[1, 0]))
    assert lse[0, 2] == -math.inf and lse[1, 0] == -math.inf
    rest = torch.ones(2, 4, dtype=torch.bool)
    rest[0, 2] = rest[1, 0] = False
    assert torch.all(torch.isfinite(got[rest]))


@pytest.mark.parametrize("cache", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lens,hq,hkv", SHAPES)
def test_some_scores_minus_infinity(cache, lens, hq, hkv):
    """Keys of -infinity in a channel where queries are positive: no weight, wherever they lie (whole
    shares of a row among them); +infinity: NaN."""
    k, v, table, n, q = _case(4, lens, hq, hkv, cache, cache)
    q[..., CHANNEL] = q[..., CHANNEL].abs() + 0.125
    for b, m in enumerate(lens):
        for i in range(m // 16 * 3 // 4):                # the first three quarters' pages
            k[int(table[b, i]), :, :, CHANNEL] = -math.inf
    if lens[0] > 64:
        k[int(table[0, lens[0] // 16 - 1]), 0, 3, CHANNEL] = math.inf
    got, _ = _run(k, v, table, n, q)
    want, _, _ = attention(k, v, table, n.tolist(), q, D ** -0.5)
    _finite_alike(got, want)


@pytest.mark.parametrize("cache", ["bf16", "f16", "f32"])
def test_capped_infinite_scores(cache):
    """cap tanh(+-infinity / cap) is +-cap."""
    k, v, table, n, q = _case(5, [100, 700], 4, 2, cache, cache)
    q[..., CHANNEL] = q[..., CHANNEL].abs() + 0.125
    k[int(table[0, 2]), :, 5, CHANNEL] = math.inf
    k[int(table[1, 3]), :, 7, CHANNEL] = -math.inf
    got, lse = _run(k, v, table, n, q, softcap=3.0)
    want, want_lse, _ = attention(k, v, table, n.tolist(), q, D ** -0.5, cap=3.0)
    assert torch.all(torch.isfinite(want))
    _finite_alike(got, want)
    # (a score: 128 products' roundings, 128 2^-24 sum |q k| scale, that sum below 23; some ulps more)
    assert torch.all((lse.double() - want_lse).abs() <= (128 * 2.0 ** -24 * 23 + 2.0 ** -17) * (1 + want_lse.abs()))


@pytest.mark.parametrize("cache,qtype", [("bf16", "f32"), ("bf16", "f16"), ("f16", "f32"), ("f16", "bf16")])
def test_infinite_queries_of_another_type(cache, qtype):
    k, v, table, n, q = _case(6, [50, 3, 1000], 4, 2, cache, qtype)
    q[:, 1, CHANNEL] = math.inf
    got, _ = _run(k, v, table, n, q)
    assert torch.all(torch.isnan(got[:, 1])) and torch.all(torch.isfinite(got[:, [0, 2, 3]]))


@pytest.mark.parametrize("hq", [8, 32])
def test_joined_every_score_minus_infinity(hq):
    """Rows wholly in pages, split between both, wholly compressed and empty."""
    B, H, page = 4, 8, 16
    n, m = [0, 200, 130, 0], [400, 40, 0, 0]
    w = workload(2, n_tokens=256, batch=B)
    cal = [ora.calibrate(w.calib(h, "k"), 4.0) for h in range(H)]
    rb, params = cal[0].record_bytes, device_params(cal)
    kc, vc = record_cache(H, 256, rb, batch=B), tile_cache(H, 256, rb, batch=B)
    ka, va = alpha_cache(H, 256, batch=B), alpha_cache(H, 256, batch=B)
    g = torch.Generator().manual_seed(11)
    x = torch.randn(256, H, D, generator=g).to(torch.bfloat16).cuda()
    for b in range(B):
        if n[b]:
            P.aatc_encode(params, H, x, n[b], H * D, P.LAYOUT_RECORDS, kc[b], ka[b], 256, 0)
            P.aatc_encode(params, H, x, n[b], H * D, P.LAYOUT_TILES, vc[b], va[b], 256, 0)
    kp, vp = (pool(g, 100, H, page, torch.bfloat16) for _ in range(2))
    kp[..., CHANNEL] = -kp[..., CHANNEL].abs() - 0.125
    table = torch.arange(100).reshape(4, 25).int().cuda()
    q = torch.randn(B, hq, D, generator=g).to(torch.bfloat16)
    ws = torch.zeros(P.aatc_decode_paged_workspace_bytes(B, hq, H, 256), dtype=torch.uint8, device="cuda")

    def run(queries):
        out = torch.full((B, hq, D), 5.0, device="cuda")
        P.aatc_decode_attention_paged(params, params, B, hq, H, queries.cuda(), kc, ka, vc, va,
                                      torch.tensor(n).int().cuda(), 256, rb, rb, D ** -0.5,
                                      P.PagedCache(kp.cuda(), vp.cuda()), table,
                                      torch.tensor(m).int().cuda(), out, ws)
        return out.cpu()
    before = run(q)
    assert torch.all(torch.isfinite(before))
    q[:, 0, CHANNEL] = math.inf
    got = run(q)
    assert torch.all(torch.isnan(got[:3, 0]))
    assert torch.all(got[3] == 0)
    # (the other heads: the compressed path's own errors, 2e-5)
    assert (got[:, 1:] - before[:, 1:]).norm() <= 2e-5 * before[:, 1:].norm()


@pytest.mark.parametrize("cache", ["bf16", "f16", "f32"])
def test_caps_past_every_score(cache):
    """A cap as large as float32 allows is none."""
    case = _case(7, [100, 900], 4, 2, cache, cache)
    want, want_lse = _run(*case)
    for cap in (1e25, 9e29, 1e30, 1e38, 3.4e38):
        got, lse = _run(*case, softcap=cap)
        _finite_alike(got, want.double())
        assert torch.all((lse - want_lse).abs() <= 2.0 ** -20 * (1 + want_lse.abs()))
