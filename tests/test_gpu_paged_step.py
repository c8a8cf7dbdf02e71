"""The paged operators together, as a serving loop uses them: rotate and append, attend over pages
alone and joined with the compressed cache, fork with copies on write, compact, compress pages, on a
stream of the caller and in a captured graph."""
import numpy as np
import pytest
import torch

import paper_2608_14191_amd as P
from helpers import alpha_cache, device_params, record_cache, rel_l2, tile_cache
from kvsynth import workload
from oracle import aatc as ora
from paged_ref import pool, turn

pytestmark = pytest.mark.gpu
D = 128
SCALE = D ** -0.5


def _compressed(B, H, n, bits=4.0):
    """Calibrations and caches of B sequences of n tokens (those below n[b] are valid), and the
    dequantized keys and values [B][H][n][D] in float64."""
    w = workload(2, n_tokens=max(n), batch=B)
    cal_k = [ora.calibrate(w.calib(h, "k"), bits) for h in range(H)]
    cal_v = [ora.calibrate(w.calib(h, "v"), bits) for h in range(H)]
    cap = -(-max(n) // 64) * 64
    rk, rv = cal_k[0].record_bytes, cal_v[0].record_bytes
    pk, pv = device_params(cal_k), device_params(cal_v)
    kc, vc = record_cache(H, cap, rk, batch=B), tile_cache(H, cap, rv, batch=B)
    ka, va = alpha_cache(H, cap, batch=B), alpha_cache(H, cap, batch=B)
    keys, values = [], []
    for b in range(B):
        x = {}
        for kind, p, cal, codes, alpha, layout, to in (
                ("k", pk, cal_k, kc, ka, P.LAYOUT_RECORDS, keys), ("v", pv, cal_v, vc, va, P.LAYOUT_TILES, values)):
            raw = np.stack([w.cache(b, h, kind, n=max(n)) for h in range(H)], axis=1)
            x[kind] = torch.from_numpy(raw.view(np.int16).copy()).view(torch.bfloat16).cuda()
            if n[b]:
                P.aatc_encode(p, H, x[kind], n[b], H * D, layout, codes[b], alpha[b], cap, 0)
            back = []
            for h in range(H):
                rec, al, _ = ora.encode(w.as_f32(w.cache(b, h, kind, n=max(n))), cal[h])
                back.append(ora.decode_tokens(rec, al, cal[h]))
            to.append(np.stack(back))
    return pk, pv, kc, ka, vc, va, rk, rv, cap, np.stack(keys), np.stack(values)


@pytest.mark.parametrize("cache_type", [torch.bfloat16, torch.float32, torch.float16])
@pytest.mark.parametrize("qtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq", [8, 32])
def test_compressed_cache_and_pages_joined(cache_type, qtype, hq):
    """Sequences that are wholly compressed, wholly in pages, split between both, and empty."""
    H, page = 8, 16
    n, m = [700, 0, 300, 0, 130], [0, 900, 333, 0, 1]
    B = len(n)
    pk, pv, kc, ka, vc, va, rk, rv, cap, keys, values = _compressed(B, H, n)
    g = torch.Generator().manual_seed(7)
    per_row = -(-max(m) // page)
    kp, vp = (pool(g, B * per_row, H, page, cache_type) for _ in range(2))
    table = torch.randperm(B * per_row, generator=g).reshape(B, per_row).int()
    q = (torch.randn(B, hq, D, generator=g) * 0.5).to(qtype)
    want = np.zeros((B, hq, D))
    for b in range(B):
        t = torch.arange(m[b])
        at, slot = table[b].long()[t // page], t % page
        for j in range(hq):
            h = j // (hq // H)
            k = np.concatenate([keys[b, h, :n[b]], kp[at, h, slot].double().numpy()])
            v = np.concatenate([values[b, h, :n[b]], vp[at, h, slot].double().numpy()])
            if len(k):
                z = k @ q[b, j].double().numpy() * SCALE
                p = np.exp(z - z.max())
                want[b, j] = (p / p.sum()) @ v
    ws = torch.zeros(P.aatc_decode_paged_workspace_bytes(B, hq, H, cap), dtype=torch.uint8, device="cuda")
    out = torch.full((B, hq, D), float("nan"), device="cuda")
    cache = P.PagedCache(kp.cuda(), vp.cuda())
    for _ in range(2):
        P.aatc_decode_attention_paged(
            pk, pv, B, hq, H, q.cuda(), kc, ka, vc, va, torch.tensor(n).int().cuda(), cap, rk, rv,
            SCALE, cache, table.cuda(), torch.tensor(m).int().cuda(), out, ws)
        got = out.cpu().numpy()
        assert np.all(got[3] == 0)
        # Wholly in pages: as the attention over pages alone.  With compressed tokens: that path's
        # own errors (its fixed-point scores and weights, T_V in two bf16 terms: 2^-16), 2e-5.
        assert rel_l2(got[1], want[1]) <= 2e-6
        for b in (0, 2, 4):
            assert rel_l2(got[b], want[b]) <= 2e-5, b


def _loop(rows, hq, hkv, page, dtype, steps, stream=None, graph=False):
    """`steps` decode steps of `rows` sequences that begin with a prompt each; returns outputs of
    every step and the whole history (rotated keys, values) for the reference."""
    g = torch.Generator().manual_seed(rows)
    per_row, n_pages = 8, rows * 8 + 4
    cache_k, cache_v = (pool(g, n_pages, hkv, page, dtype, fill=float("nan")) for _ in range(2))
    kp, vp = cache_k.cuda(), cache_v.cuda()
    cache = P.PagedCache(kp, vp)
    freq, _ = P.aatc_rope_frequencies(D, 10000.0)
    freq = torch.from_numpy(freq)
    rope = P.Rope(freq.cuda(), P.ROPE_HALF)
    table = torch.full((rows, per_row), -1, dtype=torch.int32, device="cuda")
    ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    held = torch.zeros(rows, dtype=torch.int32, device="cuda")
    pairs = torch.empty(rows, 2, dtype=torch.int32, device="cuda")
    lacking = torch.empty(1, dtype=torch.int32, device="cuda")
    space = torch.empty(P.aatc_pages_workspace_bytes(rows, n_pages), dtype=torch.uint8, device="cuda")
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(rows, hq, hkv), dtype=torch.uint8, device="cuda")
    # prompts
    lens = [5 + 17 * b % 60 for b in range(rows)]
    total = sum(lens)
    qkv = torch.randn(total, hq + 2 * hkv, D, generator=g).to(dtype)
    seq = torch.repeat_interleave(torch.arange(rows), torch.tensor(lens)).int()
    pos = torch.cat([torch.arange(n) for n in lens]).int()
    wanted = torch.tensor(lens, dtype=torch.int32, device="cuda")
    P.aatc_pages_reserve(table, ref, page, held, wanted, pairs, lacking, space)
    dev, stride = qkv.cuda(), (hq + 2 * hkv) * D
    P.aatc_paged_append(cache, table, total, dev[:, hq:hq + hkv], dev[:, hq + hkv:], stride, stride,
                        seq.cuda(), pos.cuda(), rope=rope)
    held.copy_(wanted)
    torch.cuda.synchronize()
    assert int(lacking) == 0
    history = [(seq, pos, qkv)]
    # the step's buffers
    x = torch.zeros(rows, hq + 2 * hkv, D, dtype=dtype, device="cuda")
    q = torch.zeros(rows, hq, D, dtype=dtype, device="cuda")
    out = torch.zeros(rows, hq, D, device="cuda")

    def step():
        torch.add(held, 1, out=wanted)
        P.aatc_pages_reserve(table, ref, page, held, wanted, pairs, lacking, space)
        P.aatc_paged_append(cache, table, rows, x[:, hq:hq + hkv], x[:, hq + hkv:], stride, stride,
                            None, held, rope=rope, n_q_heads=hq, q=x[:, :hq], q_tok_stride=stride,
                            q_out=q, q_out_tok_stride=hq * D)
        held.copy_(wanted)
        P.aatc_paged_decode_attention(cache, table, held, rows, hq, q, SCALE, out, ws)

    outs = []
    news = [torch.randn(rows, hq + 2 * hkv, D, generator=g).to(dtype) for _ in range(steps)]
    captured = None
    if graph:
        saved = [t.clone() for t in (held, table, ref)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        for t, s in zip((held, table, ref), saved):
            t.copy_(s)
        torch.cuda.synchronize()
    for new in news:
        n = [int(v) for v in held.tolist()]
        history.append((torch.arange(rows).int(), torch.tensor(n).int(), new))
        x.copy_(new.cuda())
        if captured is not None:
            captured.replay()
        elif stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                step()
            torch.cuda.current_stream().wait_stream(stream)
        else:
            step()
        torch.cuda.synchronize()
        assert int(lacking) == 0
        outs.append((out.cpu().double(), q.cpu(), held.tolist()))
    return outs, history, freq, (kp, vp, cache, table, ref)


def _reference(history, freq, rows, hq, hkv, upto, dtype):
    """Rotated keys (rounded to the cache's type) and values per row after history[:upto]."""
    k = [[] for _ in range(rows)]
    v = [[] for _ in range(rows)]
    for seq, pos, qkv in history[:upto]:
        kr = turn(qkv[:, hq:hq + hkv], pos, freq, 1.0, False).to(dtype)
        for t, b in enumerate(seq.tolist()):
            k[b].append(kr[t])
            v[b].append(qkv[t, hq + hkv:])
    return [torch.stack(x) for x in k], [torch.stack(x) for x in v]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("way", ["plain", "stream", "graph"])
def test_serving_loop(dtype, way):
    rows, hq, hkv, page, steps = 5, 8, 2, 8, 6
    outs, history, freq, _ = _loop(rows, hq, hkv, page, dtype, steps,
                                   stream=torch.cuda.Stream() if way == "stream" else None,
                                   graph=way == "graph")
    for i, (out, q, held) in enumerate(outs):
        k, v = _reference(history, freq, rows, hq, hkv, i + 2, dtype)
        for b in range(rows):
            assert len(k[b]) == held[b]
            for j in range(hq):
                h = j // (hq // hkv)
                z = (k[b][:, h].double() @ q[b, j].double()) * SCALE
                want = torch.softmax(z, 0) @ v[b][:, h].double()
                # a key may round to the cache's other neighbour (half an ulp either way of its
                # own): z moves by at most sum |q k| 2^-8 scale (bf16), and that for few channels
                eps = 2e-3 if dtype == torch.bfloat16 else 2e-6
                assert (out[b, j] - want).norm() <= eps * want.norm()


def test_graph_equals_eager_and_replays():
    a, _, _, _ = _loop(7, 8, 2, 8, torch.bfloat16, 8)
    b, _, _, _ = _loop(7, 8, 2, 8, torch.bfloat16, 8, graph=True)
    for (x, qx, hx), (y, qy, hy) in zip(a, b):
        assert torch.equal(x, y) and torch.equal(qx, qy) and hx == hy


def test_fork_write_compact_and_compress():
    """Fork rows, let parents and children write on, compact the pool, free the parents: attention
    sees each row's own tokens throughout; token-major pages are inputs of aatc_encode."""
    rows, hq, hkv, page = 3, 8, 8, 16
    n_pages, per_row = 64, 6
    g = torch.Generator().manual_seed(2)
    # both pools of one layer in one tensor [K, V][page][token][KV head][D]
    pools = torch.zeros(2, n_pages, page, hkv, D, dtype=torch.bfloat16, device="cuda")
    cache = P.PagedCache(pools[0].transpose(1, 2), pools[1].transpose(1, 2))
    table = torch.full((6, per_row), -1, dtype=torch.int32, device="cuda")
    ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    held = torch.zeros(6, dtype=torch.int32, device="cuda")
    pairs = torch.empty(6, 2, dtype=torch.int32, device="cuda")
    lacking = torch.empty(1, dtype=torch.int32, device="cuda")
    space = torch.empty(P.aatc_pages_workspace_bytes(6, n_pages), dtype=torch.uint8, device="cuda")
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(6, hq, hkv), dtype=torch.uint8, device="cuda")
    tokens = {b: ([], []) for b in range(6)}

    def write(counts):
        wanted = held.clone()
        for b, c in counts.items():
            wanted[b] += c
        P.aatc_pages_reserve(table, ref, page, held, wanted, pairs, lacking, space)
        assert int(lacking) == 0
        P.aatc_pages_copy(pools, pairs)
        seq = torch.tensor([b for b, c in counts.items() for _ in range(c)]).int()
        pos = torch.tensor([int(held[b]) + i for b, c in counts.items() for i in range(c)]).int()
        x = torch.randn(len(seq), 2 * hkv, D, generator=g).to(torch.bfloat16)
        for t, b in enumerate(seq.tolist()):
            tokens[b][0].append(x[t, :hkv])
            tokens[b][1].append(x[t, hkv:])
        dev = x.cuda()
        P.aatc_paged_append(cache, table, len(seq), dev[:, :hkv], dev[:, hkv:], 2 * hkv * D,
                            2 * hkv * D, seq.cuda(), pos.cuda())
        held.copy_(wanted)

    def look():
        q = torch.randn(6, hq, D, generator=g).to(torch.bfloat16)
        out = torch.empty(6, hq, D, device="cuda")
        P.aatc_paged_decode_attention(cache, table, held, 6, hq, q.cuda(), SCALE, out, ws)
        got = out.cpu().double()
        for b in range(6):
            if not tokens[b][0]:
                assert torch.all(got[b] == 0)
                continue
            k, v = torch.stack(tokens[b][0]).double(), torch.stack(tokens[b][1]).double()
            for j in range(hq):
                want = torch.softmax(k[:, j] @ q[b, j].double() * SCALE, 0) @ v[:, j]
                assert (got[b, j] - want).norm() <= 2e-6 * want.norm(), (b, j)
        t = table.cpu()
        assert torch.equal(ref.cpu(), torch.bincount(t[t >= 0].long(), minlength=n_pages).int())

    write({0: 37, 1: 16, 2: 70})
    look()
    # children 3 and 4 of row 0 (which shares a begun page), 5 of row 1 (whose pages are full)
    P.aatc_pages_fork(table, table, ref, torch.tensor([[0, 3], [0, 4], [1, 5]]).int().cuda())
    for child, parent in ((3, 0), (4, 0), (5, 1)):
        held[child] = held[parent]
        tokens[child] = (list(tokens[parent][0]), list(tokens[parent][1]))
    look()
    write({0: 1, 3: 2, 4: 30, 5: 5})
    look()
    write({1: 3, 3: 1, 2: 1})
    look()
    P.aatc_pages_free(table, ref, torch.tensor([0, 2]).int().cuda())
    for b in (0, 2):
        held[b] = 0
        tokens[b] = ([], [])
    look()
    moves = torch.empty(1, dtype=torch.int32, device="cuda")
    plan = torch.empty(n_pages // 2, 2, dtype=torch.int32, device="cuda")
    P.aatc_pages_compact(table, ref, table, ref, plan, moves, space)
    P.aatc_pages_copy(pools, plan, n_pairs=moves)
    live = int((ref > 0).sum())
    assert int(moves) > 0 and torch.all(ref[:live] > 0) and torch.all(ref[live:] == 0)
    look()
    write({1: 20, 4: 9})
    look()
    # a page's tokens compressed from where they lie, and from a copy: the same codes
    w = workload(2, n_tokens=64)
    cal = [ora.calibrate(w.calib(h, "k"), 4.0) for h in range(hkv)]
    pk, rk = device_params(cal), cal[0].record_bytes
    at = int(table[1, 0])
    codes, alpha = record_cache(hkv, 64, rk), alpha_cache(hkv, 64)
    P.aatc_encode(pk, hkv, pools[0, at], page, hkv * D, P.LAYOUT_RECORDS, codes, alpha, 64, 0)
    again, beta = record_cache(hkv, 64, rk), alpha_cache(hkv, 64)
    P.aatc_encode(pk, hkv, torch.stack(tokens[1][0][:page]).cuda(), page, hkv * D, P.LAYOUT_RECORDS,
                  again, beta, 64, 0)
    assert torch.equal(codes, again) and torch.equal(alpha, beta)


def test_joined_attention_in_a_graph():
    """Captured once, replayed with other lengths and queries, with eager calls between."""
    B, H, hq, page = 2, 8, 16, 32
    pk, pv, kc, ka, vc, va, rk, rv, cap, _, _ = _compressed(B, H, [200, 333])
    g = torch.Generator().manual_seed(9)
    kp, vp = (pool(g, 40, H, page, torch.bfloat16).cuda() for _ in range(2))
    cache = P.PagedCache(kp, vp)
    table = torch.randperm(40, generator=g).reshape(2, 20).int().cuda()
    n, m = torch.tensor([200, 333]).int().cuda(), torch.tensor([600, 7]).int().cuda()
    q = torch.randn(B, hq, D, generator=g).cuda()
    spaces = [torch.zeros(P.aatc_decode_paged_workspace_bytes(B, hq, H, cap), dtype=torch.uint8, device="cuda")
              for _ in range(2)]
    outs = [torch.zeros(B, hq, D, device="cuda") for _ in range(2)]

    def call(i):
        P.aatc_decode_attention_paged(pk, pv, B, hq, H, q, kc, ka, vc, va, n, cap, rk, rv, SCALE, cache,
                                      table, m, outs[i], spaces[i])
    call(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0)
    for lens, pages in (([200, 333], [600, 7]), ([0, 100], [640, 0]), ([1, 64], [0, 129]), ([200, 0], [33, 0])):
        n.copy_(torch.tensor(lens).int())
        m.copy_(torch.tensor(pages).int())
        q.copy_(torch.randn(B, hq, D, generator=g))
        outs[0].fill_(float("nan"))
        graph.replay()
        call(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.all(torch.isfinite(outs[0]))
