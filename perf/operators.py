"""Performance cases of the paged cache at input precision and of the operators around it.

A serving program keeps the tokens that are not compressed (whole short sequences, the recent
window, layers left as they are) in pages of a pool: page i of a cache holds `page` consecutive
tokens of one sequence, for every KV head, and a sequence's row of the page table names its
pages in order (negative: no page there, its tokens are not attended).

`case["kind"]`:
  rope     rotary positions of queries or keys (aatc_rope), or the inverse rotation;
  append   new tokens: rotate q and k, store k and v in the sequences' pages
           (aatc_paged_append);
  attend   attention of one new token per sequence over its pages
           (aatc_paged_decode_attention);
  fork     release the children of the step before, fork children from their parents' rows, get
           them a page to write to, copy what they share (aatc_pages_free, _fork, _reserve,
           _copy);
  compact  move the used pages to the pool's front (aatc_pages_compact, aatc_pages_copy).
"""
import math

import torch

own = False

D = 128
SCALE = D ** -0.5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------------------
def _rope(tokens, heads, rot, layout, dtype, **more):
    return dict(dict(kind="rope", tokens=tokens, heads=heads, rot=rot, layout=layout, dtype=dtype,
                     scaled=False, inverse=False, first=0), **more)


def _append(rows, tokens, hq, hkv, dtype, cache, **more):
    return dict(dict(kind="append", rows=rows, tokens=tokens, hq=hq, hkv=hkv, dtype=dtype,
                     cache=cache, rot=D, layout="half", scaled=False, page=16, order="head",
                     length=1024, padded=False), **more)


def _attend(batch, hq, hkv, n, cache, **more):
    return dict(dict(kind="attend", batch=batch, hq=hq, hkv=hkv, n=n, cache=cache,
                     dtype="bf16" if cache == "bf16" else "f32", page=16, order="head",
                     ragged=batch > 1, window=0, sink=0, cap=0.0, slopes=False, lse=False), **more)


def _fork(parents, children, pages, pools, page, page_bytes):
    return dict(kind="fork", parents=parents, children=children, pages=pages, pools=pools,
                page=page, page_bytes=page_bytes)


def _compact(pages, used, rows, pools, page_bytes):
    return dict(kind="compact", pages=pages, used=used, rows=rows, pools=pools,
                page_bytes=page_bytes)


def listed():
    return [
        # The queries of a 4096-token prompt, the Llama-3.1-8B layer's 32 heads.
        dict(_rope(4096, 32, D, "half", "bf16"), name="rope_prompt_4k"),
        # Keys of a long prompt far behind the trained positions, half of each head rotated in
        # interleaved pairs, float32, turned back to position 0 (the gradient's direction too).
        dict(_rope(65536, 8, 64, "interleaved", "f32", scaled=True, inverse=True, first=400000),
             name="rope_keys_back_64k"),
        # One decoded token of each of 64 sequences: the launch counts.
        dict(_append(64, 64, 32, 8, "bf16", "bf16"), name="append_step_b64"),
        # Prompts of different lengths, padded, into token-major pages of float16.
        dict(_append(5, 16384, 28, 4, "f32", "f16", layout="interleaved", rot=96, scaled=True,
                     page=64, order="token", length=8192, padded=True), name="append_prompts_16k"),
        # A short conversation, not worth compressing yet: latency only.
        dict(_attend(1, 32, 8, 300, "bf16"), name="attend_b1_300"),
        # The headline length of the compressed path, uncompressed, float16.
        dict(_attend(1, 32, 8, 32768, "f16", dtype="f16", page=64), name="attend_b1_32k"),
        # A serving batch of the Qwen-2.5-7B shape, sequences of different lengths.
        dict(_attend(8, 28, 4, 16384, "bf16", lse=True), name="attend_qwen_b8_16k"),
        # Many conversations, float32 token-major pages, a window and a sink with the pages in
        # between given back, capped scores and a distance bias.
        dict(_attend(48, 16, 8, 5000, "f32", order="token", page=32, window=2048, sink=4, cap=30.0,
                     slopes=True), name="attend_window_b48"),
        # Long contexts: the memory's rate counts.
        dict(_attend(4, 32, 8, 131072, "bf16", page=128, ragged=False), name="attend_b4_128k"),
        # Beam search over one prompt: four beams' pages in eight pools.
        dict(_fork(4, 4, 40, 8, 16, 32768), name="fork_beams_4"),
        # Several samples for each of 32 prompts, sixteen pools.
        dict(_fork(32, 128, 24, 16, 32, 65536), name="fork_samples_128"),
        # A pool of 4096 pages, half of them free in between, before a resize.
        dict(_compact(4096, 0.5, 64, 8, 32768), name="compact_4k_pages"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attend", "attend", "attend", "fork", "compact"])
    rot = rng.choice([D, D, 96, 64, 32, 50, 2])
    layout = rng.choice(["half", "interleaved"])
    scaled = rng.random() < 0.4
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "rope":
        heads = rng.choice([1, 4, 8, 28, 32, 64])
        return _rope(_log_int(rng, 1, 65536 * 8 // heads), heads, rot, layout, dtype,
                     scaled=scaled, inverse=rng.random() < 0.3,
                     first=rng.choice([0, rng.randint(0, 1000000)]))
    if kind == "append":
        hq, hkv = rng.choice([(32, 8), (28, 4), (64, 8), (16, 8), (8, 8)])
        rows = _log_int(rng, 1, 256)
        tokens = rows if rng.random() < 0.5 else _log_int(rng, rows, max(rows, 16384))
        return _append(rows, tokens, hq, hkv, dtype, rng.choice(["bf16", "f16", "f32"]), rot=rot,
                       layout=layout, scaled=scaled, page=rng.choice([8, 16, 32, 64, 256]),
                       order=rng.choice(["head", "token"]),
                       length=max(2 * tokens // rows, _log_int(rng, 16, 4096)),
                       padded=tokens > rows and rng.random() < 0.5)
    if kind == "attend":
        hq, hkv = rng.choice([(32, 8), (28, 4), (64, 8), (16, 8), (8, 8), (40, 2), (20, 4)])
        batch = _log_int(rng, 1, 256)
        cache = rng.choice(["bf16", "bf16", "f16", "f32"])
        n = _log_int(rng, 1, min(131072, (65536 if cache == "f32" else 131072) * 32 // (batch * hkv)))
        window = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
        return _attend(batch, hq, hkv, n, cache, dtype=rng.choice([cache, "f32", "bf16"]),
                       page=rng.choice([8, 16, 32, 64, 128]), order=rng.choice(["head", "token"]),
                       window=window, sink=rng.choice([0, 4, 33]) if window else 0,
                       cap=rng.choice([0.0, 0.0, 20.0, 50.0]), slopes=rng.random() < 0.25,
                       lse=rng.random() < 0.5)
    if kind == "fork":
        parents = _log_int(rng, 1, 64)
        return _fork(parents, rng.randint(1, 128), rng.randint(1, 24), rng.randint(1, 16),
                     rng.choice([8, 16, 32]), 16 * _log_int(rng, 8, 4096))
    return _compact(_log_int(rng, 64, 8192), rng.choice([0.1, 0.3, 0.5, 0.8, 0.95]),
                    rng.randint(1, 64), rng.randint(1, 8), 16 * _log_int(rng, 8, 2048))


# ---------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _frequencies(rot, scaled):
    """Angles per position of the rot / 2 pairs, base 500000; scaled: slow pairs 8 times slower,
    fast ones kept, a line between (by how often a pair turns in 8192 positions)."""
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaled:
        turns = 8192 * f / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (keep + (1 - keep) / 8.0)
    return f.cuda()


def _tokens(g, shape, gain=None):
    """Values of queries, keys or values: normal, with a head's channels of falling spread, and a
    few outlier channels for keys."""
    x = torch.randn(*shape, generator=g, device="cuda")
    spread = (1.0 + torch.arange(D, device="cuda")) ** -0.25 * 1.5
    if gain:
        spread = spread.clone()
        spread[torch.randint(0, D, (4,), generator=g, device="cuda")] *= gain
    return x.mul_(spread[torch.randperm(D, generator=g, device="cuda")])


def _lengths(g, count, most, ragged):
    """Sequence lengths: all `most`, or between a third of it and it (one of them `most`)."""
    n = torch.full((count,), most, device="cuda", dtype=torch.int32)
    if ragged:
        n = (most * (1 + 2 * torch.rand(count, generator=g, device="cuda")) / 3).ceil().to(torch.int32)
        n[torch.randint(0, count, (1,), generator=g, device="cuda")] = most
    return n


def _pool(n_pages, hkv, page, dtype, order, fill):
    """A pool's pages, seen as [page][KV head][token][channel] whatever their order in memory."""
    if order == "head":
        return torch.full((n_pages, hkv, page, D), fill, device="cuda", dtype=dtype)
    return torch.full((n_pages, page, hkv, D), fill, device="cuda", dtype=dtype).transpose(1, 2)


def prepare(case, seed):
    g = _generator(seed)
    return dict(rope=_prepare_rope, append=_prepare_append, attend=_prepare_attend,
                fork=_prepare_fork, compact=_prepare_compact)[case["kind"]](dict(case), g)


def _rope_handle(s):
    if own:
        import paper_2608_14191_amd as P
        layout = P.ROPE_HALF if s["layout"] == "half" else P.ROPE_INTERLEAVED
        s["rope"] = P.Rope(s["freq"], layout, s["factor"])


def _cache_handle(s):
    if own:
        import paper_2608_14191_amd as P
        s["cache"] = P.PagedCache(s["k_pages"], s["v_pages"])


def _prepare_rope(s, g):
    s["x"] = _tokens(g, (s["tokens"], s["heads"], D)).to(TYPES[s["dtype"]])
    s["out"] = torch.empty_like(s["x"])
    s["pos"] = s["first"] + torch.randperm(s["tokens"], generator=g, device="cuda").to(torch.int32)
    s["freq"], s["factor"] = _frequencies(s["rot"], s["scaled"]), 1.2 if s["scaled"] else 1.0
    _rope_handle(s)
    return s


def _prepare_append(s, g):
    rows, tokens, page, hq, hkv = s["rows"], s["tokens"], s["page"], s["hq"], s["hkv"]
    # `tokens` new tokens, dealt to the rows in runs, each after what its row holds already
    each = tokens // rows
    cut = torch.arange(1, rows, device="cuda") * tokens // rows + torch.randint(
        0, each, (rows - 1,), generator=g, device="cuda")
    seq = torch.searchsorted(cut, torch.arange(tokens, device="cuda"), right=True)
    new = torch.bincount(seq, minlength=rows)
    held = torch.randint(0, s["length"], (rows,), generator=g, device="cuda")
    start = torch.cumsum(new, 0) - new
    pos = held[seq] + torch.arange(tokens, device="cuda") - start[seq]
    if s["padded"]:                    # the last tokens of the batch are padding
        pos[tokens - tokens // 8:] = -1
    per_row = -(-(s["length"] + 2 * each + 2) // page)
    n_pages = rows * per_row + 3
    s["table"] = torch.randperm(n_pages, generator=g, device="cuda")[:rows * per_row] \
        .reshape(rows, per_row).to(torch.int32)
    s["seq"], s["pos"] = seq.to(torch.int32), pos.to(torch.int32)
    x = torch.cat([_tokens(g, (tokens, hq, D)), _tokens(g, (tokens, hkv, D), 8.0),
                   _tokens(g, (tokens, hkv, D))], 1).to(TYPES[s["dtype"]])
    s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]   # one projection's
    s["q_out"] = torch.zeros(tokens, hq, D, device="cuda", dtype=TYPES[s["dtype"]])
    s["k_pages"] = _pool(n_pages, hkv, page, TYPES[s["cache"]], s["order"], 0.5)
    s["v_pages"] = _pool(n_pages, hkv, page, TYPES[s["cache"]], s["order"], 0.5)
    s["freq"], s["factor"] = _frequencies(s["rot"], s["scaled"]), 1.2 if s["scaled"] else 1.0
    _rope_handle(s)
    _cache_handle(s)
    return s


def _prepare_attend(s, g):
    batch, page, hq, hkv, n = s["batch"], s["page"], s["hq"], s["hkv"], s["n"]
    s["len"] = _lengths(g, batch, n, s["ragged"])
    if s["ragged"] and batch > 2:
        s["len"][1 if int(s["len"][1]) < n else 2] = 0       # a slot without a sequence
    per_row = -(-n // page)
    n_pages = batch * per_row + 3
    s["table"] = torch.randperm(n_pages, generator=g, device="cuda")[:batch * per_row] \
        .reshape(batch, per_row).to(torch.int32)
    dtype = TYPES[s["cache"]]
    for name, gain in (("k_pages", 8.0), ("v_pages", None)):
        # (a few pages' values at a time: the pool in float32 would take twice its size more)
        pool = _pool(n_pages, hkv, page, dtype, s["order"], 0.0)
        few = max(1, (1 << 26) // (hkv * page * D))
        for i in range(0, n_pages, few):
            m = min(few, n_pages - i)
            pool[i:i + m] = _tokens(g, (m, hkv, page, D), gain)
        s[name] = pool
    # what lies behind a sequence's end, and in pages no sequence has, is of no value
    t = torch.arange(per_row * page, device="cuda").reshape(per_row, page)
    past = (t >= s["len"][:, None, None]).nonzero(as_tuple=True)
    for name in ("k_pages", "v_pages"):
        s[name][s["table"].long()[past[0], past[1]], :, past[2]] = float("nan")
    if s["window"]:                    # pages behind the sink and before the window are given back
        first = torch.arange(per_row, device="cuda") * page
        gone = (first >= s["sink"]) & (first + page <= s["len"][:, None] - s["window"])
        s["table"][gone] = -1
    s["q"] = (_tokens(g, (batch, hq, D)) * 0.7).to(TYPES[s["dtype"]])
    s["slope"] = torch.logspace(-1, -8, hq, base=2.0, device="cuda") if s["slopes"] else None
    s["out"] = torch.empty(batch, hq, D, device="cuda")
    s["lse_out"] = torch.empty(batch, hq, device="cuda") if s["lse"] else None
    _cache_handle(s)
    if own:
        import paper_2608_14191_amd as P
        s["workspace"] = torch.zeros(P.aatc_paged_decode_workspace_bytes(batch, hq, hkv),
                                     dtype=torch.uint8, device="cuda")
    return s


def _prepare_fork(s, g):
    parents, children, page = s["parents"], s["children"], s["page"]
    per_row = s["pages"] + 1
    rows = parents + children
    n_pages = parents * s["pages"] + 2 * children + 5
    length = torch.randint((s["pages"] - 1) * page + 1, s["pages"] * page + 1, (parents,),
                           generator=g, device="cuda")
    free = torch.randperm(n_pages, generator=g, device="cuda")
    s["table"] = torch.full((rows, per_row), -1, device="cuda", dtype=torch.int32)
    s["table"][:parents, :-1] = free[:parents * s["pages"]].reshape(parents, -1).to(torch.int32)
    s["ref"] = torch.zeros(n_pages, device="cuda", dtype=torch.int32)
    s["ref"][s["table"][:parents, :-1].long()] = 1
    parent = torch.randint(0, parents, (children,), generator=g, device="cuda")
    child = parents + torch.arange(children, device="cuda")
    s["children_rows"] = child.to(torch.int32)
    s["forks"] = torch.stack([parent, child], 1).to(torch.int32).contiguous()
    held = torch.zeros(rows, device="cuda", dtype=torch.int32)
    held[:parents], held[parents:] = length.to(torch.int32), length[parent].to(torch.int32)
    s["held"], s["wanted"] = held, held.clone()
    s["wanted"][parents:] += 1                                     # a token more for each child
    s["pools_data"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (s["pools"], n_pages, s["page_bytes"] // 4),
                                    generator=g, device="cuda", dtype=torch.int32)
    s["pairs"] = torch.empty(rows, 2, device="cuda", dtype=torch.int32)
    s["short"] = torch.empty(1, device="cuda", dtype=torch.int32)
    if own:
        import paper_2608_14191_amd as P
        s["workspace"] = torch.empty(P.aatc_pages_workspace_bytes(rows, n_pages),
                                     dtype=torch.uint8, device="cuda")
    return s


def _prepare_compact(s, g):
    n_pages, rows = s["pages"], s["rows"]
    used = max(1, int(n_pages * s["used"]))
    per_row = -(-used // rows)
    ids = torch.randperm(n_pages, generator=g, device="cuda")[:used].to(torch.int32)
    flat = torch.full((rows * per_row,), -1, device="cuda", dtype=torch.int32)
    flat[:used] = ids
    s["table"] = flat.reshape(rows, per_row)
    if rows > 1:                       # the last row shares the first one's first page
        s["table"][-1, 0] = s["table"][0, 0]
    s["ref"] = torch.bincount(s["table"][s["table"] >= 0].long(), minlength=n_pages).to(torch.int32)
    s["pools_data"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (s["pools"], n_pages, s["page_bytes"] // 4),
                                    generator=g, device="cuda", dtype=torch.int32)
    s["new_table"], s["new_ref"] = torch.empty_like(s["table"]), torch.empty_like(s["ref"])
    s["pairs"] = torch.empty(n_pages // 2, 2, device="cuda", dtype=torch.int32)
    s["moves"] = torch.empty(1, device="cuda", dtype=torch.int32)
    if own:
        import paper_2608_14191_amd as P
        s["workspace"] = torch.empty(P.aatc_pages_workspace_bytes(rows, n_pages),
                                     dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------
def run(s):
    return (globals()["_own_" + s["kind"]] if own else globals()["_plain_" + s["kind"]])(s)


def _own_rope(s):
    import paper_2608_14191_amd as P
    P.aatc_rope(s["x"], s["tokens"], s["heads"], s["heads"] * D, s["pos"], s["rope"], s["out"],
                s["heads"] * D, inverse=s["inverse"])
    return s["out"]


def _own_append(s):
    import paper_2608_14191_amd as P
    stride = (s["hq"] + 2 * s["hkv"]) * D
    P.aatc_paged_append(s["cache"], s["table"], s["tokens"], s["k"], s["v"], stride, stride,
                        s["seq"], s["pos"], rope=s["rope"], n_q_heads=s["hq"], q=s["q"],
                        q_tok_stride=stride, q_out=s["q_out"], q_out_tok_stride=s["hq"] * D)
    return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}


def _own_attend(s):
    import paper_2608_14191_amd as P
    P.aatc_paged_decode_attention(s["cache"], s["table"], s["len"], s["batch"], s["hq"], s["q"],
                                  SCALE, s["out"], s["workspace"], lse=s["lse_out"],
                                  window=s["window"], sink=s["sink"], softcap=s["cap"],
                                  slopes=s["slope"])
    return {"out": s["out"], "lse": s["lse_out"]} if s["lse"] else {"out": s["out"]}


def _own_fork(s):
    import paper_2608_14191_amd as P
    P.aatc_pages_free(s["table"], s["ref"], s["children_rows"])
    P.aatc_pages_fork(s["table"], s["table"], s["ref"], s["forks"])
    P.aatc_pages_reserve(s["table"], s["ref"], s["page"], s["held"], s["wanted"], s["pairs"],
                         s["short"], s["workspace"])
    P.aatc_pages_copy(s["pools_data"], s["pairs"])
    return {k: s[k] for k in ("table", "ref", "pairs", "short", "pools_data")}


def _own_compact(s):
    import paper_2608_14191_amd as P
    P.aatc_pages_compact(s["table"], s["ref"], s["new_table"], s["new_ref"], s["pairs"],
                         s["moves"], s["workspace"])
    P.aatc_pages_copy(s["pools_data"], s["pairs"], n_pairs=s["moves"])
    return {k: s[k] for k in ("new_table", "new_ref", "pairs", "moves", "pools_data")}


# The plain forms.
def _plain_turn(x, pos, freq, factor, layout, inverse=False):
    """x [tokens][heads][D] rotated, in float32 (the angles in float64)."""
    rot = 2 * freq.numel()
    angle = pos.double()[:, None] * freq
    c, s = (factor * angle.cos()).float()[:, None], (factor * angle.sin()).float()[:, None]
    s = -s if inverse else s
    x = x.float()
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., rot:]], -1)
    a, b = x[..., :rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., rot:]], -1)


def _plain_rope(s):
    return _plain_turn(s["x"], s["pos"], s["freq"], s["factor"], s["layout"],
                       s["inverse"]).to(TYPES[s["dtype"]])


def _plain_append(s):
    t = (s["pos"] >= 0).nonzero()[:, 0]
    pos, seq = s["pos"].long()[t], s["seq"].long()[t]
    at, slot = s["table"].long()[seq, pos // s["page"]], pos % s["page"]
    turn = lambda x: _plain_turn(x, pos, s["freq"], s["factor"], s["layout"])    # noqa: E731
    s["q_out"][t] = turn(s["q"][t]).to(TYPES[s["dtype"]])
    s["k_pages"][at, :, slot] = turn(s["k"][t]).to(TYPES[s["cache"]])
    s["v_pages"][at, :, slot] = s["v"][t].float().to(TYPES[s["cache"]])
    return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}


def _plain_rows(pages, table):
    """The sequences' tokens [batch][KV head][token][D] in float32 (any page where none is)."""
    x = pages[table.clamp(min=0).long()]
    return x.transpose(1, 2).flatten(2, 3).float()


def _plain_attend(s):
    batch, hkv, n = s["batch"], s["hkv"], s["len"][:, None]
    t = torch.arange(s["table"].shape[1] * s["page"], device="cuda")[None]
    on = (t < n) & (s["table"] >= 0).repeat_interleave(s["page"], 1)
    if s["window"]:
        on = on & ((t >= n - s["window"]) | (t < s["sink"]))
    q = s["q"].float().reshape(batch, hkv, -1, D)
    z = torch.matmul(q, _plain_rows(s["k_pages"], s["table"]).transpose(2, 3)) * SCALE
    if s["cap"]:
        z = s["cap"] * torch.tanh(z / s["cap"])
    if s["slopes"]:
        z = z - s["slope"].reshape(1, hkv, -1, 1) * (n - 1 - t)[:, None, None].float()
    z = torch.where(on[:, None, None], z, -math.inf)
    top = z.amax(3, keepdim=True)
    p = torch.exp(z - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(3, keepdim=True)
    v = torch.where(on[:, None, :, None], _plain_rows(s["v_pages"], s["table"]), 0.0)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    out = {"out": o.reshape(batch, -1, D)}
    if s["lse"]:
        out["lse"] = (top + total.log()).reshape(batch, -1)
    return out


def _plain_fork(s):
    table, ref, page = s["table"], s["ref"], s["page"]
    # the children's pages of the step before go back
    old = table[s["children_rows"].long()]
    ref.index_add_(0, old.clamp(min=0).long().flatten(), -(old >= 0).int().flatten())
    # the children take their parents' pages
    new = table[s["forks"][:, 0].long()]
    table[s["forks"][:, 1].long()] = new
    ref.index_add_(0, new.clamp(min=0).long().flatten(), (new >= 0).int().flatten())
    # rows that grow: a copy of a partial last page that others hold too, unless no row after it
    # would be left to hold it, and the pages that the new tokens need (one at most here)
    rows = torch.arange(table.shape[0], device="cuda")
    first, last = (s["held"] + page - 1) // page, (s["wanted"] + page - 1) // page
    grows = s["wanted"] > s["held"]
    partial = grows & (s["held"] % page > 0)
    at = (s["held"] // page).clamp(max=table.shape[1] - 1).long()
    shared = torch.where(partial, table[rows, at], -1 - rows.int())
    earlier = ((shared[:, None] == shared[None]) & (rows[:, None] > rows[None])).sum(1)
    copy = partial & (ref[shared.clamp(min=0).long()] - earlier > 1)
    want = copy | (grows & (last > first))
    free = torch.sort((ref > 0).int(), stable=True)[1]
    got = free[(torch.cumsum(want, 0) - 1).clamp(min=0)].int()
    s["short"][0] = (want.sum() - (ref <= 0).sum()).clamp(min=0)
    table[rows, at] = torch.where(want, got, table[rows, at])
    ref.index_add_(0, shared.clamp(min=0).long(), -copy.int())
    ref.index_add_(0, got.long(), want.int())
    s["pairs"][:] = torch.where(copy[:, None], torch.stack([shared, got], 1), -1)
    # the contents
    pair = s["pairs"][copy].long()
    s["pools_data"][:, pair[:, 1]] = s["pools_data"][:, pair[:, 0]]
    return {k: s[k] for k in ("table", "ref", "pairs", "short", "pools_data")}


def _plain_compact(s):
    ref, n_pages = s["ref"], s["pages"]
    ids = torch.arange(n_pages, device="cuda", dtype=torch.int32)
    live = ref > 0
    front = ids < live.sum()
    src, dst = ids[live & ~front], ids[~live & front]              # as many of one as of the other
    to = ids.clone()
    to[src.long()] = dst
    s["new_table"][:] = torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], s["table"])
    s["new_ref"][:] = torch.where(front, ref, 0)
    s["new_ref"][dst.long()] = ref[src.long()]
    s["pairs"].fill_(-1)
    s["pairs"][:src.numel()] = torch.stack([src, dst], 1)
    s["moves"].fill_(src.numel())
    s["pools_data"][:, dst.long()] = s["pools_data"][:, src.long()]
    return {k: s[k] for k in ("new_table", "new_ref", "pairs", "moves", "pools_data")}


# ---------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------
def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    c = case
    if c["kind"] == "rope":
        n = c["tokens"] * c["heads"]
        return {"bytes": 2 * n * D * _size(c["dtype"]) + 4 * c["tokens"], "flops": 3 * n * c["rot"]}
    if c["kind"] == "append":
        n = c["tokens"] - (c["tokens"] // 8 if c["padded"] else 0)
        moved = (2 * c["hq"] + 2 * c["hkv"]) * D * _size(c["dtype"]) + 2 * c["hkv"] * D * _size(c["cache"])
        return {"bytes": n * (moved + 12), "flops": 3 * n * (c["hq"] + c["hkv"]) * c["rot"]}
    if c["kind"] == "attend":
        # (ragged lengths are two thirds of the longest in the mean)
        mean = c["n"] * (2 * c["batch"] + 1) / (3 * c["batch"]) if c["ragged"] else c["n"]
        if c["window"]:
            mean = min(mean, c["window"] + c["sink"])
        tokens = c["batch"] * mean
        ends = c["batch"] * c["hq"] * D * (_size(c["dtype"]) + 4)
        return {"bytes": 2 * tokens * c["hkv"] * D * _size(c["cache"]) + ends + 4 * tokens / c["page"],
                "flops": 4 * tokens * c["hq"] * D}
    if c["kind"] == "fork":
        # a child's page is copied where its parent's last page is not full
        copies = c["children"] * (c["page"] - 1) / c["page"]
        return {"bytes": 2 * copies * c["pools"] * c["page_bytes"] + 12 * c["children"] * c["pages"],
                "flops": 0}
    used = max(1, int(c["pages"] * c["used"]))
    moved = used * (c["pages"] - used) / c["pages"]
    return {"bytes": 2 * moved * c["pools"] * c["page_bytes"] + 16 * c["pages"], "flops": 0}


# ---------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------
def _exact_turn(x, pos, freq, factor, layout, back):
    """x [tokens][heads][D] as complex numbers times factor exp(+-i pos freq)."""
    rot = 2 * freq.numel()
    x = x.double().clone()
    lo = slice(0, rot // 2) if layout == "half" else slice(0, rot, 2)
    hi = slice(rot // 2, rot) if layout == "half" else slice(1, rot, 2)
    a = torch.outer(pos.double(), freq)[:, None]
    w = torch.complex(x[..., lo], x[..., hi]) * torch.polar(torch.full_like(a, factor), -a if back else a)
    x[..., lo], x[..., hi] = w.real, w.imag
    return x


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None                    # nothing computed: whole numbers and moved bytes
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_turn(s["x"], s["pos"], s["freq"], s["factor"], s["layout"], s["inverse"])
    if case["kind"] == "append":
        out = {"q": s["q_out"].double(), "k": s["k_pages"].double(), "v": s["v_pages"].double()}
        t = torch.nonzero(s["pos"] >= 0).flatten()
        pos, seq = s["pos"].long()[t], s["seq"].long()[t]
        at, slot = s["table"].long()[seq, pos // s["page"]], pos % s["page"]
        for name in ("q", "k"):
            turned = _exact_turn(s[name][t], pos, s["freq"], s["factor"], s["layout"], False)
            if name == "q":
                out["q"][t] = turned
            else:
                out["k"][at, :, slot] = turned
        out["v"][at, :, slot] = s["v"][t].double()
        return out
    batch, hq, hkv, page = s["batch"], s["hq"], s["hkv"], s["page"]
    out = torch.zeros(batch, hq, D, device="cuda", dtype=torch.float64)
    lse = torch.full((batch, hq), -math.inf, device="cuda", dtype=torch.float64)
    table, lens = s["table"].tolist(), s["len"].tolist()
    for b, n in enumerate(lens):
        t = [i for i in range(n) if table[b][i // page] >= 0 and
             (not s["window"] or i >= n - s["window"] or i < s["sink"])]
        if not t:
            continue
        at = torch.tensor(t, device="cuda")
        pages, slot = s["table"][b].long()[at // page], at % page
        for h in range(hkv):
            mine = slice(h * hq // hkv, (h + 1) * hq // hkv)
            k, v = s["k_pages"][pages, h, slot].double(), s["v_pages"][pages, h, slot].double()
            z = (k @ s["q"][b, mine].double().T) * SCALE
            if s["cap"]:
                z = s["cap"] * torch.tanh(z / s["cap"])
            if s["slopes"]:
                z = z - s["slope"][mine].double() * (n - 1 - at).double()[:, None]
            lse[b, mine] = torch.logsumexp(z, 0)
            out[b, mine] = torch.softmax(z, 0).T.contiguous() @ v
    return {"out": out, "lse": lse} if s["lse"] else {"out": out}
