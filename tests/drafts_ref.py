"""Plain 64-bit forms of the drafted tokens' operators and of sparse attention, on the CPU, for the GPU
tests."""
import math

import torch

D = 128


def families(parent, m):
    """[draft] -> its ancestors and itself, in order; parent: a list, or None for a chain."""
    kin = []
    for i in range(m):
        up = i - 1 if parent is None else parent[i]
        kin.append((kin[up] if 0 <= up < i else []) + [i])
    return kin


def softmax_rows(z, v):
    """(output, log-sum-exp, sum p |v|) of scores z [tokens] over v [tokens][D], float64."""
    if len(z) == 0:
        return torch.zeros(D, dtype=torch.float64), -math.inf, torch.zeros(D, dtype=torch.float64)
    p = torch.softmax(z, 0)
    return p @ v, torch.logsumexp(z, 0), p @ v.abs()


def tree_attention(k_pages, v_pages, table, lens, q, scale, n_draft=None, parent=None, window=0,
                   sink=0, cap=0.0, slopes=None):
    """(out, lse, spread) of q [batch][drafts][heads][D]; rows without a draft are NaN."""
    n_pages, hkv, page, _ = k_pages.shape
    batch, drafts, hq, _ = q.shape
    most = table.shape[1] * page
    out = torch.full((batch, drafts, hq, D), math.nan, dtype=torch.float64)
    spread, lse = out.clone(), torch.full((batch, drafts, hq), math.nan, dtype=torch.float64)
    for b in range(batch):
        n = min(max(int(lens[b]), 0), most)
        m = drafts if n_draft is None else min(max(int(n_draft[b]), 0), drafts)
        kin = families(None if parent is None else parent[b].tolist(), m)
        row = table[b].tolist()
        there = [t // page < len(row) and 0 <= row[t // page] < n_pages for t in range(n + m)]
        for i in range(m):
            here = n + len(kin[i]) - 1
            both = [(t, t) for t in range(n)] + [(n + j, n + d) for d, j in enumerate(kin[i])]
            both = [(t, pos) for t, pos in both if there[t] and
                    (window == 0 or pos > here - window or t < sink)]
            t = torch.tensor([x for x, _ in both], dtype=torch.long)
            far = here - torch.tensor([pos for _, pos in both], dtype=torch.float64)
            pages, slot = table[b].long()[t // page], t % page
            for h in range(hkv):
                k, v = k_pages[pages, h, slot].double(), v_pages[pages, h, slot].double()
                for j in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                    z = (k @ q[b, i, j].double()) * scale
                    if cap:
                        z = cap * torch.tanh(z / cap)
                    if slopes is not None:
                        z = z - slopes[j].double() * far
                    out[b, i, j], lse[b, i, j], spread[b, i, j] = softmax_rows(z, v)
    return out, lse, spread


def accept(parent, drafted, chosen, m):
    """(path, next) of one sequence; lists."""
    if m == 0:
        return [], -1
    path = [0]
    while True:
        now = path[-1]
        up = [i - 1 if parent is None else parent[i] for i in range(m)]
        step = [i for i in range(now + 1, m) if up[i] == now and drafted[i] == chosen[now]]
        if not step:
            return path, chosen[now]
        path.append(step[0])


def step_of(top):
    """Exponent of the smallest power of two, from 2^-50 on, of which 127 reach top."""
    if top == 0:
        return -50
    m, e = math.frexp(top)
    return max(-50, e - 7 if m <= 127 / 128 else e - 6)


def page_bounds(keys):
    """(codes [2][D], scale) of the keys [tokens][D] of a page and KV head."""
    k = keys.double()
    top = k.abs().max().item()
    if not math.isfinite(top) or top > 127 * 2.0 ** 100:
        return torch.zeros(2, D, dtype=torch.int8), math.inf
    s = 2.0 ** step_of(top)
    return torch.stack([torch.ceil(k.amax(0) / s), torch.floor(k.amin(0) / s)]).to(torch.int8), s


def picked_pages(q, codes, scales, row, n, page, n_pages, most, first, last, scale):
    """Table indexes that one KV head's queries q [heads][D] pick; codes [n_pages][2][D]."""
    pages = -(-n // page)
    there = [i for i in range(pages) if 0 <= row[i] < n_pages]
    says = []
    for x in q.double() * (-1 if scale < 0 else 1):
        if torch.isfinite(x).all():
            e = step_of(x.abs().max().item())
            says.append((e, torch.round(x / 2.0 ** e)))
    at = torch.tensor([row[i] for i in there], dtype=torch.long)
    hi, lo = codes[at, 0].double(), codes[at, 1].double()
    best = torch.full((len(there),), 0.0 if not says else -math.inf, dtype=torch.float64)
    for e, u in says:
        s = torch.maximum(u * hi, u * lo).sum(1) * 2.0 ** max(-60, e - max(x for x, _ in says))
        best = torch.maximum(best, s)
    step = scales[at].double()
    best = torch.where(torch.isinf(step), math.inf, best * torch.where(torch.isinf(step), 1.0, step))
    rank = {}
    for i, s in zip(there, best.tolist()):
        rank[i] = (0 if i < first or i >= pages - last else 1, -s, i)
    return sorted(sorted(there, key=lambda i: rank[i])[:most])


def sparse_attention(k_pages, v_pages, codes, scales, table, lens, q, scale, most, first, last,
                     cap=0.0):
    """(picked [batch][KV head] lists, out, lse, spread)."""
    n_pages, hkv, page, _ = k_pages.shape
    batch, hq, _ = q.shape
    out = torch.zeros(batch, hq, D, dtype=torch.float64)
    spread, lse = out.clone(), torch.zeros(batch, hq, dtype=torch.float64)
    picked = []
    for b in range(batch):
        n = min(max(int(lens[b]), 0), table.shape[1] * page)
        row = table[b].tolist()
        picked.append([])
        for h in range(hkv):
            mine = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            some = picked_pages(q[b, mine], codes[:, h], scales[:, h], row, n, page, n_pages, most,
                                first, last, scale)
            picked[b].append(some)
            t = torch.tensor([t for i in some for t in range(i * page, min(n, (i + 1) * page))],
                             dtype=torch.long)
            pages, slot = table[b].long()[t // page], t % page
            k, v = k_pages[pages, h, slot].double(), v_pages[pages, h, slot].double()
            for j in range(mine.start, mine.stop):
                z = (k @ q[b, j].double()) * scale
                if cap:
                    z = cap * torch.tanh(z / cap)
                out[b, j], lse[b, j], spread[b, j] = softmax_rows(z, v)
    return picked, out, lse, spread
