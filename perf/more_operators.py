"""Performance cases of drafted tokens and of sparse attention over the paged cache.

Speculative decoding: a step brings a tree of drafted tokens per sequence, stored in the slots
behind the sequence's tokens.  Draft i attends the whole sequence, itself and its ancestors.  What
the model then chooses after each draft says which path of the tree is accepted; its keys and
values move up to the sequence's end.

Sparse attention: every page and KV head keeps each key channel's largest and smallest value in
8 bits.  They bound what any key of the page can score, and each sequence and KV head attends the
pages of the highest bounds only.

`case["kind"]`:
  tree     attention of a tree of drafted tokens over pages (aatc_paged_tree_attention);
  accept   the accepted path of each tree, and its tokens moved, in every layer
           (aatc_paged_tree_accept);
  bounds   the bounds of the pages that new tokens fell into (aatc_page_bounds);
  sparse   pages chosen by their bounds, attention of one new token per sequence over them
           (aatc_paged_sparse_attention).
"""
import math

import numpy as np
import torch

own = False

D = 128
SCALE = D ** -0.5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------------------
def _tree(batch, hq, hkv, n, drafts, cache, **more):
    return dict(dict(kind="tree", batch=batch, hq=hq, hkv=hkv, n=n, drafts=drafts, cache=cache,
                     dtype="bf16" if cache == "bf16" else "f32", page=16, order="head",
                     ragged=batch > 1, chain=False, window=0, sink=0, cap=0.0, slopes=False,
                     lse=False), **more)


def _accept(batch, hkv, n, drafts, layers, cache, **more):
    return dict(dict(kind="accept", batch=batch, hkv=hkv, n=n, drafts=drafts, layers=layers,
                     cache=cache, page=16, order="head"), **more)


def _bounds(rows, hkv, n, new, cache, **more):
    return dict(dict(kind="bounds", rows=rows, hkv=hkv, n=n, new=new, cache=cache, page=16,
                     order="head"), **more)


def _sparse(batch, hq, hkv, n, most, cache, **more):
    return dict(dict(kind="sparse", batch=batch, hq=hq, hkv=hkv, n=n, most=most, cache=cache,
                     dtype="bf16" if cache == "bf16" else "f32", page=16, order="head",
                     ragged=batch > 1, first=1, last=2, cap=0.0, lse=False), **more)


def listed():
    return [
        # A short conversation, a few drafts: latency only.
        dict(_tree(1, 32, 8, 300, 8, "bf16"), name="tree_b1_300_8"),
        # One long sequence of the Llama-3.1-8B layer, the widest tree: the matrix products count.
        dict(_tree(1, 32, 8, 32768, 64, "f16", dtype="f16", page=64), name="tree_b1_32k_64"),
        # A serving batch of the Qwen-2.5-7B shape, sequences and trees of different sizes.
        dict(_tree(8, 28, 4, 16384, 26, "bf16", lse=True), name="tree_qwen_b8_26"),
        # Many conversations, four tokens ahead in a chain, float32 token-major pages, a window
        # and a sink, capped scores and a distance bias.
        dict(_tree(48, 16, 8, 5000, 5, "f32", order="token", page=32, chain=True, window=2048,
                   sink=4, cap=30.0, slopes=True), name="tree_window_b48_5"),
        # The last tokens of a very long prompt: the memory's rate counts.
        dict(_tree(1, 32, 8, 131072, 16, "bf16", chain=True, page=128), name="chunk_b1_128k_16"),
        # One sequence, one layer's pools: the launch counts.
        dict(_accept(1, 8, 1000, 8, 1, "bf16"), name="accept_b1_8"),
        # A serving batch, every layer at once.
        dict(_accept(64, 8, 500, 32, 32, "bf16"), name="accept_b64_32"),
        # One decoded token of each of 64 sequences: its page's bounds anew.
        dict(_bounds(64, 8, 4096, 1, "bf16"), name="bounds_step_b64"),
        # A whole prompt's pages, float32, token-major.
        dict(_bounds(1, 8, 65536, 65536, "f32", page=32, order="token"), name="bounds_prompt_64k"),
        # The headline length, 1024 of 32768 tokens attended: latency.
        dict(_sparse(1, 32, 8, 32768, 64, "f16", dtype="f16"), name="sparse_b1_32k_64"),
        # A ragged serving batch, float32 queries, token-major pages, capped scores.
        dict(_sparse(32, 28, 4, 8192, 32, "bf16", dtype="f32", page=32, order="token", cap=50.0,
                     lse=True), name="sparse_qwen_b32_32"),
        # Long contexts, 4096 of 131072 tokens attended: the bounds of 8192 pages are read.
        dict(_sparse(4, 32, 8, 131072, 256, "bf16", ragged=False), name="sparse_b4_128k_256"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "accept", "bounds", "sparse", "sparse"])
    hq, hkv = rng.choice([(32, 8), (28, 4), (64, 8), (16, 8), (8, 8), (40, 2), (20, 4)])
    cache = rng.choice(["bf16", "bf16", "f16", "f32"])
    dtype = rng.choice([cache, "f32", "bf16"])
    order = rng.choice(["head", "token"])
    page = rng.choice([8, 16, 32, 64, 128])
    tokens = (4 if cache == "f32" else 8) * 131072 // hkv        # of all sequences together
    if kind == "tree":
        batch = _log_int(rng, 1, 64)
        drafts = _log_int(rng, 1, 64)
        n = _log_int(rng, 1, max(1, min(131072, tokens // batch, 60000000 // (batch * drafts * hq))))
        window = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
        return _tree(batch, hq, hkv, n, drafts, cache, dtype=dtype, page=page, order=order,
                     chain=rng.random() < 0.3, window=window,
                     sink=rng.choice([0, 4, 33]) if window else 0,
                     cap=rng.choice([0.0, 0.0, 20.0, 50.0]), slopes=rng.random() < 0.25,
                     lse=rng.random() < 0.5)
    if kind == "accept":
        batch = _log_int(rng, 1, 128)
        layers = _log_int(rng, 1, 32)
        drafts = _log_int(rng, 1, 64)
        small = rng.choice([8, 16, 32])
        return _accept(batch, rng.choice([1, 4, 8]), _log_int(rng, 1, 1000), drafts,
                       min(layers, 1 + 1024 // (batch * (1 + drafts // small))), cache, page=small,
                       order=order)
    if kind == "bounds":
        rows = _log_int(rng, 1, 128)
        n = _log_int(rng, 1, min(131072, tokens // (2 * rows)))
        new = n if rng.random() < 0.5 else rng.randint(1, n)
        return _bounds(rows, hkv, n, new, cache, page=page, order=order)
    batch = _log_int(rng, 1, 64)
    n = _log_int(rng, 1, min(131072, tokens // (2 * batch)))
    most = _log_int(rng, 4, max(4, 4096 // page))
    return _sparse(batch, hq, hkv, n, most, cache, dtype=dtype, page=page, order=order,
                   first=rng.choice([0, 1]), last=rng.choice([1, 2, 3]),
                   cap=rng.choice([0.0, 0.0, 20.0, 50.0]), lse=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


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


def _pools(s, g, n_pages, layers=0):
    """Key and value pages, seen as [page][KV head][token][channel] whatever their order."""
    hkv, page, dtype = s["hkv"], s["page"], TYPES[s["cache"]]
    lead = (layers,) if layers else ()
    for name, gain in (("k_pages", 8.0), ("v_pages", None)):
        if s["order"] == "head":
            pool = torch.empty(*lead, n_pages, hkv, page, D, device="cuda", dtype=dtype)
        else:
            pool = torch.empty(*lead, n_pages, page, hkv, D, device="cuda", dtype=dtype)
        # (a few pages' values at a time: the pool in float32 would take twice its size more)
        flat = pool.view(-1, hkv * page, D)
        few = max(1, (1 << 26) // (hkv * page * D))
        for i in range(0, flat.shape[0], few):
            m = min(few, flat.shape[0] - i)
            flat[i:i + m] = _tokens(g, (m, hkv * page, D), gain)
        s[name] = pool if s["order"] == "head" else pool.transpose(-3, -2)


def _table(g, rows, per_row):
    """Rows of pages in random order, out of a few more than there are."""
    n_pages = rows * per_row + 3
    table = torch.randperm(n_pages, generator=g, device="cuda")[:rows * per_row]
    return table.reshape(rows, per_row).to(torch.int32), n_pages


def _nothing_behind(s, end):
    """What lies behind the sequences' ends is of no value."""
    per_row, page = s["table"].shape[1], s["page"]
    t = torch.arange(per_row * page, device="cuda").reshape(per_row, page)
    past = (t >= end[:, None, None]).nonzero(as_tuple=True)
    for name in ("k_pages", "v_pages"):
        s[name][s["table"].long()[past[0], past[1]], :, past[2]] = float("nan")


def prepare(case, seed):
    g = _generator(seed)
    return dict(tree=_prepare_tree, accept=_prepare_accept, bounds=_prepare_bounds,
                sparse=_prepare_sparse)[case["kind"]](dict(case), g)


def _cache_handle(s):
    if own:
        import paper_2608_14191_amd as P
        s["cache"] = P.PagedCache(s["k_pages"], s["v_pages"])


def _trees(s, g):
    """Parents: the draft before, or one of the four before."""
    batch, drafts = s["batch"], s["drafts"]
    i = torch.arange(drafts, device="cuda")
    back = torch.randint(1, 5, (batch, drafts), generator=g, device="cuda")
    s["parent"] = torch.where(i > 0, (i - back).clamp(min=0), -1).to(torch.int32).contiguous()


def _prepare_tree(s, g):
    batch, page, hq, hkv, n, drafts = (s[k] for k in ("batch", "page", "hq", "hkv", "n", "drafts"))
    s["len"] = _lengths(g, batch, n, s["ragged"])
    s["n_draft"] = None
    if s["ragged"]:                    # trees of different sizes, and a slot without a sequence
        s["n_draft"] = _lengths(g, batch, drafts, True)
        if batch > 2:
            gone = 1 if int(s["len"][1]) < n else 2
            s["len"][gone], s["n_draft"][gone] = 0, 0
    if s["chain"]:
        s["parent"] = None
    else:
        _trees(s, g)
    s["table"], n_pages = _table(g, batch, -(-(n + drafts) // page))
    _pools(s, g, n_pages)
    _nothing_behind(s, s["len"] + (drafts if s["n_draft"] is None else s["n_draft"]))
    if s["window"]:                    # pages behind the sink and before the window are given back
        first = torch.arange(s["table"].shape[1], device="cuda") * page
        gone = (first >= s["sink"]) & (first + page <= s["len"][:, None] - s["window"])
        s["table"][gone] = -1
    # the queries are part of one projection's output
    x = (_tokens(g, (batch * drafts, hq + 2 * hkv, D)) * 0.7).to(TYPES[s["dtype"]])
    s["q"] = x[:, :hq]
    s["slope"] = torch.logspace(-1, -8, hq, base=2.0, device="cuda") if s["slopes"] else None
    s["out"] = torch.zeros(batch, drafts, hq, D, device="cuda")
    s["lse_out"] = torch.zeros(batch, drafts, hq, device="cuda") if s["lse"] else None
    _cache_handle(s)
    if own:
        import paper_2608_14191_amd as P
        s["workspace"] = torch.zeros(P.aatc_paged_tree_workspace_bytes(batch, drafts, hq, hkv),
                                     dtype=torch.uint8, device="cuda")
    return s


def _prepare_accept(s, g):
    batch, drafts, page, n = s["batch"], s["drafts"], s["page"], s["n"]
    s["len"] = _lengths(g, batch, n, batch > 1)
    s["n_draft"] = _lengths(g, batch, drafts, batch > 1)
    _trees(s, g)
    # every draft's token, and the model's choice after it: mostly one of its children's
    s["drafted"] = torch.randint(0, 100000, (batch, drafts), generator=g, device="cuda").to(torch.int32)
    agrees = torch.rand(batch, drafts, generator=g, device="cuda") < 0.9
    agrees[:, 0] = False
    i = torch.arange(drafts, device="cuda").expand(batch, -1)
    child = torch.full((batch, drafts), drafts, device="cuda")
    child.scatter_reduce_(1, s["parent"].long().clamp(min=0), torch.where(agrees, i, drafts), "amin")
    other = torch.randint(0, 100000, (batch, drafts), generator=g, device="cuda").to(torch.int32)
    s["chosen"] = torch.where(child < drafts,
                              torch.gather(s["drafted"], 1, child.clamp(max=drafts - 1)), other)
    # only the pages that the drafts lie in: those before are the same one
    per_row = -(-(n + drafts) // page)
    held = 2 + drafts // page
    own_pages, n_pages = _table(g, batch, held)
    at = torch.arange(per_row, device="cuda") - (s["len"][:, None] // page)
    s["table"] = torch.gather(own_pages, 1, at.clamp(0, held - 1).long())
    s["table"][(at < 0) | (at >= held)] = -1
    _pools(s, g, n_pages, s["layers"])
    s["path"] = torch.empty(batch, drafts, device="cuda", dtype=torch.int32)
    for name in ("accepted", "next", "len_out"):
        s[name] = torch.empty(batch, device="cuda", dtype=torch.int32)
    if own:
        import paper_2608_14191_amd as P
        s["cache"] = P.PagedCache(s["k_pages"][0], s["v_pages"][0])
    return s


def _prepare_bounds(s, g):
    rows, page, n = s["rows"], s["page"], s["n"]
    s["wanted"] = _lengths(g, rows, n, rows > 1)
    s["held"] = (s["wanted"] - s["new"]).clamp(min=0)
    s["table"], n_pages = _table(g, rows, -(-n // page))
    _pools(s, g, n_pages)
    _nothing_behind(s, s["wanted"])
    s["codes"] = torch.zeros(n_pages, s["hkv"], 2, D, device="cuda", dtype=torch.int8)
    s["scales"] = torch.zeros(n_pages, s["hkv"], device="cuda")
    _cache_handle(s)
    return s


def _prepare_sparse(s, g):
    batch, page, hq, hkv, n = s["batch"], s["page"], s["hq"], s["hkv"], s["n"]
    s["len"] = _lengths(g, batch, n, s["ragged"])
    if s["ragged"] and batch > 2:
        s["len"][1 if int(s["len"][1]) < n else 2] = 0       # a slot without a sequence
    per_row = -(-n // page)
    s["table"], n_pages = _table(g, batch, per_row)
    _pools(s, g, n_pages)
    _nothing_behind(s, s["len"])
    s["codes"] = torch.zeros(n_pages, hkv, 2, D, device="cuda", dtype=torch.int8)
    s["scales"] = torch.zeros(n_pages, hkv, device="cuda")
    first = torch.arange(per_row, device="cuda") * page
    _plain_page_bounds(s, (first < s["len"][:, None]).nonzero(as_tuple=True), s["len"])
    s["q"] = (_tokens(g, (batch, hq, D)) * 0.7).to(TYPES[s["dtype"]])
    s["out"] = torch.empty(batch, hq, D, device="cuda")
    s["lse_out"] = torch.empty(batch, hq, device="cuda") if s["lse"] else None
    s["picked"] = torch.empty(batch, hkv, s["most"], device="cuda", dtype=torch.int32)
    _cache_handle(s)
    if own:
        import paper_2608_14191_amd as P
        s["workspace"] = torch.zeros(
            P.aatc_paged_sparse_workspace_bytes(batch, hq, hkv, per_row), dtype=torch.uint8,
            device="cuda")
    return s


# ---------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------
def run(s):
    return (globals()["_own_" + s["kind"]] if own else globals()["_plain_" + s["kind"]])(s)


def _own_tree(s):
    import paper_2608_14191_amd as P
    P.aatc_paged_tree_attention(s["cache"], s["table"], s["len"], s["batch"], s["drafts"], s["hq"],
                                s["q"], SCALE, s["out"], s["workspace"], n_draft=s["n_draft"],
                                parent=s["parent"], window=s["window"], sink=s["sink"],
                                softcap=s["cap"], slopes=s["slope"], lse=s["lse_out"])
    return {"out": s["out"], "lse": s["lse_out"]} if s["lse"] else {"out": s["out"]}


def _own_accept(s):
    import paper_2608_14191_amd as P
    P.aatc_paged_tree_accept(s["cache"], s["table"], s["len"], s["batch"], s["drafts"], s["drafted"],
                             s["chosen"], s["path"], s["accepted"], s["next"], s["len_out"],
                             n_draft=s["n_draft"], parent=s["parent"], n_layers=s["layers"],
                             layer_stride=s["k_pages"].stride(0))
    return {k: s[k] for k in ("path", "accepted", "next", "len_out", "k_pages", "v_pages")}


def _own_bounds(s):
    import paper_2608_14191_amd as P
    P.aatc_page_bounds(s["cache"], s["table"], s["held"], s["wanted"], s["codes"], s["scales"])
    return {"codes": s["codes"], "scales": s["scales"]}


def _own_sparse(s):
    import paper_2608_14191_amd as P
    P.aatc_paged_sparse_attention(s["cache"], s["table"], s["len"], s["codes"], s["scales"],
                                  s["batch"], s["hq"], s["q"], SCALE, s["picked"], s["out"],
                                  s["workspace"], first=s["first"], last=s["last"],
                                  softcap=s["cap"], lse=s["lse_out"])
    out = {"out": s["out"], "picked": s["picked"]}
    return dict(out, lse=s["lse_out"]) if s["lse"] else out


# The plain forms.
def _plain_family(parent, batch, drafts):
    """[batch][draft][draft]: whether the second is the first or an ancestor of it."""
    eye = torch.eye(drafts, device="cuda")
    if parent is None:
        return torch.ones(drafts, drafts, device="cuda").tril().bool().expand(batch, drafts, drafts)
    up = (parent[:, :, None] == torch.arange(drafts, device="cuda")).float()
    return torch.matrix_power(eye + up, 64) > 0


def _plain_attention(s, q, k, v, on, bias):
    """q [...][queries][D], k and v [...][tokens][D] in float32: outputs and log-sum-exp of the
    tokens that are `on`, [...][queries][tokens]."""
    z = torch.matmul(q, k.transpose(-1, -2)) * SCALE
    if s["cap"]:
        z = s["cap"] * torch.tanh(z / s["cap"])
    if bias is not None:
        z = z - bias
    z = torch.where(on, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    v = torch.where(on.any(-2)[..., None], v, 0.0)
    return torch.matmul(p, v) / torch.where(total > 0, total, 1.0), (top + total.log())[..., 0]


def _plain_tree(s):
    batch, drafts, hq, hkv, page = (s[k] for k in ("batch", "drafts", "hq", "hkv", "page"))
    n = s["len"].long()[:, None]
    m = drafts if s["n_draft"] is None else s["n_draft"].long()[:, None]
    kin = _plain_family(s["parent"], batch, drafts)
    depth = kin.sum(2) - 1
    tokens = s["table"].shape[1] * page
    t = torch.arange(tokens, device="cuda")[None].expand(batch, -1)
    j = (t - n).clamp(0, drafts - 1)                               # the draft in each slot
    pos_t = torch.where(t < n, t, n + torch.gather(depth, 1, j))
    pos_q = n + depth
    mine = torch.gather(kin, 2, j[:, None].expand(-1, drafts, -1))
    on = (t < n)[:, None] | (mine & (t < n + m)[:, None])
    on = on & (s["table"] >= 0).repeat_interleave(page, 1)[:, None]
    if s["window"]:
        on = on & ((pos_t[:, None] > pos_q[:, :, None] - s["window"]) | (t < s["sink"])[:, None])
    at = s["table"].clamp(min=0).long()
    k, v = (s[x][at].transpose(1, 2).flatten(2, 3).float() for x in ("k_pages", "v_pages"))
    # queries [batch][KV head][head of its group and draft][D]
    group = hq // hkv
    q = s["q"].float().reshape(batch, drafts, hkv, group, D).permute(0, 2, 3, 1, 4).flatten(2, 3)
    bias = None
    if s["slopes"]:
        far = (pos_q[:, :, None] - pos_t[:, None]).float()[:, None, None]
        bias = (s["slope"].reshape(1, hkv, group, 1, 1) * far).flatten(2, 3)
    o, lse = _plain_attention(s, q, k, v, on[:, None].repeat(1, 1, group, 1), bias)
    o = o.reshape(batch, hkv, group, drafts, D).permute(0, 3, 1, 2, 4).reshape(batch, drafts, hq, D)
    lse = lse.reshape(batch, hkv, group, drafts).permute(0, 3, 1, 2).reshape(batch, drafts, hq)
    there = (torch.arange(drafts, device="cuda")[None] < m)[:, :, None]
    out = {"out": torch.where(there[..., None], o, s["out"])}
    if s["lse"]:
        out["lse"] = torch.where(there, lse, s["lse_out"])
    return out


def _plain_accept(s):
    batch, drafts, page = s["batch"], s["drafts"], s["page"]
    i = torch.arange(drafts, device="cuda")
    n, m, parent = s["len"].long(), s["n_draft"].long(), s["parent"].long()
    # a draft agrees if its parent's choice is its token, and no earlier child's
    same = (torch.gather(s["chosen"], 1, parent.clamp(min=0)) == s["drafted"]) & (parent >= 0)
    earlier = ((parent[:, :, None] == parent[:, None]) & same[:, None] & (i[:, None] > i)).any(2)
    agrees = (same & ~earlier) | (i == 0)
    agrees = agrees & (i < m[:, None])
    # accepted: it and its ancestors all agree
    kin = _plain_family(s["parent"], batch, drafts)
    taken = (agrees[:, None] | ~kin).all(2) & kin[:, :, 0]
    count = taken.sum(1)
    s["path"].fill_(-1)
    b, j = taken.nonzero(as_tuple=True)
    to = (torch.cumsum(taken, 1) - 1)[b, j]
    s["path"][b, to] = j.int()
    s["accepted"].copy_(count)
    last = torch.gather(s["path"].long(), 1, (count - 1).clamp(min=0)[:, None]).clamp(min=0)
    s["next"].copy_(torch.where(count > 0, torch.gather(s["chosen"], 1, last)[:, 0], -1))
    s["len_out"].copy_(n + count)
    # the accepted tokens' keys and values move up, all read before any is written
    src, dst = n[b] + j, n[b] + to
    from_page, to_page = (s["table"].long()[b, x // page] for x in (src, dst))
    for x in (s["k_pages"], s["v_pages"]):
        x[:, to_page, :, dst % page] = x[:, from_page, :, src % page]
    return {k: s[k] for k in ("path", "accepted", "next", "len_out", "k_pages", "v_pages")}


def _plain_step_of(top):
    """The smallest power of two, at least 2^-50, of which 127 reach `top` (and its exponent)."""
    m, e = torch.frexp(top)
    e = torch.where(top > 0, torch.where(m <= 127.0 / 128.0, e - 7, e - 6), -50).clamp(min=-50)
    return e


def _plain_power(e):
    """2^e in float64, exactly (a library's power may be an ulp off)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _plain_page_bounds(s, which, end):
    """The bounds of the pages `which` (rows, entries), each of its tokens before `end` [row]."""
    page = s["page"]
    row, entry = which
    t = entry[:, None] * page + torch.arange(page, device="cuda")
    on = (t < end.long()[row][:, None])[:, None, :, None]
    at = s["table"].long()[row, entry]
    k = s["k_pages"][at].float()
    hi = torch.where(on, k, -math.inf).amax(2)
    lo = torch.where(on, k, math.inf).amin(2)
    e = _plain_step_of(torch.maximum(hi, -lo).amax(2))[..., None]
    s["codes"][at, :, 0] = torch.ceil(hi.double() * _plain_power(-e)).to(torch.int8)
    s["codes"][at, :, 1] = torch.floor(lo.double() * _plain_power(-e)).to(torch.int8)
    s["scales"][at] = _plain_power(e)[..., 0].float()


def _plain_bounds(s):
    page = s["page"]
    i = torch.arange(s["table"].shape[1], device="cuda")[None] * page
    new = (i < s["wanted"][:, None]) & (i + page > s["held"][:, None])
    _plain_page_bounds(s, new.nonzero(as_tuple=True), s["wanted"])
    return {"codes": s["codes"], "scales": s["scales"]}


def _plain_sparse(s):
    batch, hq, hkv, page, most = (s[k] for k in ("batch", "hq", "hkv", "page", "most"))
    n, at = s["len"].long()[:, None], s["table"].clamp(min=0).long()
    entry = torch.arange(s["table"].shape[1], device="cuda")[None]
    pages = (n + page - 1) // page
    # queries in 8 bits, with steps relative to the group's largest
    q = s["q"].float().reshape(batch, hkv, -1, D)
    e = _plain_step_of(q.abs().amax(3))
    code = torch.round(q.double() * _plain_power(-e[..., None]))
    rel = _plain_power((e - e.amax(2, keepdim=True)).clamp(min=-60))
    # the most that a key of a page can score: whole numbers below 2^24, exact in float32
    both = torch.cat([code.clamp(min=0), code.clamp(max=0)], 3).float()
    bound = s["codes"][at].flatten(3, 4).float().permute(0, 2, 3, 1)        # [..][2 D][page]
    score = (torch.matmul(both, bound.contiguous()) * rel[..., None].float()).amax(2)
    score = score * s["scales"][at].transpose(1, 2)
    always = ((entry < s["first"]) | (entry >= pages - s["last"]))[:, None]
    there = ((entry < pages) & (s["table"] >= 0))[:, None]
    key = torch.where(there, torch.where(always, math.inf, score), -math.inf)
    order = torch.sort(key, dim=2, descending=True, stable=True)[1][:, :, :most]
    taken = torch.zeros_like(key, dtype=torch.bool).scatter_(2, order, True) & there
    b, h, i = taken.nonzero(as_tuple=True)
    s["picked"].fill_(-1)
    s["picked"][b, h, (torch.cumsum(taken, 2) - 1)[b, h, i]] = i.int()
    # attention over the tokens of the pages picked
    picked = s["picked"].long()
    t = (picked[..., None] * page + torch.arange(page, device="cuda")).flatten(2, 3)
    on = (t >= 0) & (t < n[:, :, None])
    phys = torch.gather(at[:, None].expand(-1, hkv, -1), 2, picked.clamp(min=0))
    head = torch.arange(hkv, device="cuda")[None, :, None]
    k, v = (s[x][phys, head].flatten(2, 3).float() for x in ("k_pages", "v_pages"))
    o, lse = _plain_attention(s, q, k, v, on[:, :, None].expand(-1, -1, q.shape[2], -1), None)
    out = {"out": o.reshape(batch, hq, D), "picked": s["picked"]}
    return dict(out, lse=lse.reshape(batch, hq)) if s["lse"] else out


# ---------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------
def _size(name):
    return 4 if name == "f32" else 2


def _mean(count, most, ragged):
    """Ragged lengths are two thirds of the longest in the mean."""
    return most * (2 * count + 1) / (3 * count) if ragged else most


def work(case):
    c = case
    if c["kind"] == "tree":
        mean = _mean(c["batch"], c["n"], c["ragged"])
        if c["window"]:
            mean = min(mean, c["window"] + c["sink"])
        drafts = _mean(c["batch"], c["drafts"], c["ragged"])
        tokens = c["batch"] * (mean + drafts)
        ends = c["batch"] * drafts * c["hq"] * D * (_size(c["dtype"]) + 4)
        return {"bytes": 2 * tokens * c["hkv"] * D * _size(c["cache"]) + ends + 4 * tokens / c["page"],
                "flops": 4 * tokens * drafts * c["hq"] * D}
    if c["kind"] == "accept":
        # (three to four drafts are accepted, of which those behind a gap move)
        moved = c["batch"] * 1.6 * (c["drafts"] - 1) / (c["drafts"] + 6)
        return {"bytes": 4 * moved * c["layers"] * c["hkv"] * D * _size(c["cache"]) +
                16 * c["batch"] * c["drafts"], "flops": 0}
    if c["kind"] == "bounds":
        mean = _mean(c["rows"], c["n"], c["rows"] > 1)
        tokens = c["rows"] * min(mean, c["new"] + (c["page"] - 1) / 2)
        return {"bytes": tokens * c["hkv"] * D * _size(c["cache"]) +
                max(tokens / c["page"], c["rows"]) * (c["hkv"] * (2 * D + 4) + 4),
                "flops": 2 * tokens * c["hkv"] * D}
    mean = _mean(c["batch"], c["n"], c["ragged"])
    pages = c["batch"] * -(-mean // c["page"])
    tokens = c["batch"] * min(mean, c["most"] * c["page"])
    ends = c["batch"] * c["hq"] * D * (_size(c["dtype"]) + 4) + 4 * c["batch"] * c["hkv"] * c["most"]
    return {"bytes": pages * (c["hkv"] * (2 * D + 4) + 4) + ends +
            2 * tokens * c["hkv"] * D * _size(c["cache"]),
            "flops": 4 * pages * c["hq"] * D + 4 * tokens * c["hq"] * D}


# ---------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------
def _exact_rows(s, b, h, at, q, slope, far):
    """Output and log-sum-exp of queries q [queries][D] over tokens `at` of sequence b, KV head h."""
    pages, slot = s["table"][b].long()[at // s["page"]], at % s["page"]
    k, v = s["k_pages"][pages, h, slot].double(), s["v_pages"][pages, h, slot].double()
    z = (k @ q.double().T) * SCALE
    if s["cap"]:
        z = s["cap"] * torch.tanh(z / s["cap"])
    if slope is not None:
        z = z - slope.double() * far.double()[:, None]
    return torch.softmax(z, 0).T.contiguous() @ v, torch.logsumexp(z, 0)


def _exact_tree(s):
    batch, drafts, hq, hkv, page = (s[k] for k in ("batch", "drafts", "hq", "hkv", "page"))
    out, lse = s["out"].double(), torch.zeros(batch, drafts, hq, device="cuda", dtype=torch.float64)
    q = s["q"].reshape(batch, drafts, hq, D)
    table, lens = s["table"].tolist(), s["len"].tolist()
    m = [drafts] * batch if s["n_draft"] is None else s["n_draft"].tolist()
    parent = s["parent"].tolist() if s["parent"] is not None else [[i - 1 for i in range(drafts)]] * batch
    for b in range(batch):
        n, kin = lens[b], []
        for i in range(m[b]):
            kin.append((kin[parent[b][i]] if parent[b][i] >= 0 else []) + [i])
        for i in range(m[b]):
            here = n + len(kin[i]) - 1
            slots = list(range(n)) + [n + j for j in kin[i]]
            pos = list(range(n)) + [n + d for d in range(len(kin[i]))]
            some = [x for x, (t, p) in enumerate(zip(slots, pos)) if table[b][t // page] >= 0 and
                    (not s["window"] or p > here - s["window"] or t < s["sink"])]
            at = torch.tensor([slots[x] for x in some], device="cuda")
            far = here - torch.tensor([pos[x] for x in some], device="cuda")
            for h in range(hkv):
                mine = slice(h * hq // hkv, (h + 1) * hq // hkv)
                out[b, i, mine], lse[b, i, mine] = _exact_rows(
                    s, b, h, at, q[b, i, mine], s["slope"][mine] if s["slopes"] else None, far)
    return {"out": out, "lse": lse} if s["lse"] else {"out": out}


def _exact_bounds(s):
    """The steps of the pages' bounds (the codes are whole numbers)."""
    scales = s["scales"].double()
    held, wanted, page = s["held"].tolist(), s["wanted"].tolist(), s["page"]
    for r, (a, z) in enumerate(zip(held, wanted)):
        if a >= z:
            continue
        entry = torch.arange(a // page, (z - 1) // page + 1, device="cuda")
        at = s["table"][r].long()[entry]
        inside = entry[:, None] * page + torch.arange(page, device="cuda") < z
        top = torch.where(inside[:, None, :, None], s["k_pages"][at].double().abs(), 0.0).amax((2, 3))
        # the smallest step of which 127 reach the page's largest value
        top = top.cpu().numpy()
        e = np.maximum(np.frexp(top)[1] - 8, -50)
        for _ in range(2):
            e = np.where(np.ldexp(127.0, e) < top, e + 1, e)
        scales[at] = torch.from_numpy(np.ldexp(1.0, e)).cuda()
    return {"codes": None, "scales": scales}


def _exact_sparse(s):
    batch, hq, hkv, page = (s[k] for k in ("batch", "hq", "hkv", "page"))
    out = torch.zeros(batch, hq, D, device="cuda", dtype=torch.float64)
    lse = torch.full((batch, hq), -math.inf, device="cuda", dtype=torch.float64)
    values = s["codes"].double() * s["scales"].double()[..., None, None]
    for b, n in enumerate(s["len"].tolist()):
        pages = -(-n // page)
        if not pages:
            continue
        at = s["table"][b, :pages].long()
        for h in range(hkv):
            mine = slice(h * hq // hkv, (h + 1) * hq // hkv)
            q = s["q"][b, mine].double()
            top = q.abs().amax(1).cpu().numpy()
            e = np.frexp(top)[1] - 8
            for _ in range(2):
                e = np.where(np.ldexp(127.0, e) < top, e + 1, e)
            step = torch.from_numpy(np.ldexp(1.0, e)).cuda()[:, None]
            near = torch.round(q / step) * step
            most = torch.maximum(near[:, None] * values[at, h, 0], near[:, None] * values[at, h, 1])
            rank = most.sum(2).amax(0).tolist()
            always = [i for i in range(pages) if i < s["first"] or i >= pages - s["last"]]
            rest = sorted(set(range(pages)) - set(always), key=lambda i: (-rank[i], i))
            picked = sorted((always + rest)[:s["most"]])
            ts = torch.tensor([t for i in picked for t in range(i * page, min(n, (i + 1) * page))],
                              device="cuda")
            out[b, mine], lse[b, mine] = _exact_rows(s, b, h, ts, s["q"][b, mine], None, None)
    found = {"out": out, "picked": None}
    return dict(found, lse=lse) if s["lse"] else found


def exact(case, seed):
    if case["kind"] == "accept":
        return None                    # nothing computed: whole numbers and moved bytes
    s = prepare(case, seed)
    return dict(tree=_exact_tree, bounds=_exact_bounds, sparse=_exact_sparse)[case["kind"]](s)
