"""Plain 64-bit forms of the paged operators, on the CPU (NumPy-like torch), for the GPU tests."""
import math

import torch

D = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# Half a step of each type, relative to the value.
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}


def turn(x, pos, freq, factor, interleaved, inverse=False):
    """x [tokens][heads][D] float64 rotated."""
    rot = 2 * freq.numel()
    angle = pos.double()[:, None] * freq.double()
    c, s = factor * angle.cos()[:, None], factor * angle.sin()[:, None]
    s = -s if inverse else s
    y = x.double().clone()
    lo, hi = ((slice(0, rot, 2), slice(1, rot, 2)) if interleaved
              else (slice(0, rot // 2), slice(rot // 2, rot)))
    a, b = y[..., lo].clone(), y[..., hi].clone()
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    return y


def attended(n, row, n_pages, page, window, sink):
    """Token indexes of a sequence of n tokens with page-table row `row` (a list)."""
    return [t for t in range(n) if 0 <= row[t // page] < n_pages and
            (window == 0 or t >= n - window or t < sink)]


def attention(k_pages, v_pages, table, lens, q, scale, window=0, sink=0, cap=0.0, slopes=None):
    """(out [batch][heads][D], lse [batch][heads], weights' spread [batch][heads]) in float64;
    pages [page][KV head][token][D].  The third: sum_t p_t |v_t|, the scale of rounding errors."""
    n_pages, hkv, page, _ = k_pages.shape
    batch, hq, _ = q.shape
    most = table.shape[1] * page
    out = torch.zeros(batch, hq, D, dtype=torch.float64)
    spread = torch.zeros(batch, hq, D, dtype=torch.float64)
    lse = torch.full((batch, hq), -math.inf, dtype=torch.float64)
    for b in range(batch):
        n = min(max(int(lens[b]), 0), most)
        ts = attended(n, table[b].tolist(), n_pages, page, window, sink)
        if not ts:
            continue
        t = torch.tensor(ts)
        pages, slot = table[b].long()[t // page], t % page
        for j in range(hq):
            h = j // (hq // hkv)
            k, v = k_pages[pages, h, slot].double(), v_pages[pages, h, slot].double()
            z = (k @ q[b, j].double()) * scale
            if cap:
                z = cap * torch.tanh(z / cap)
            if slopes is not None:
                z = z - slopes[j].double() * (n - 1 - t).double()
            lse[b, j] = torch.logsumexp(z, 0)
            p = torch.softmax(z, 0)
            out[b, j], spread[b, j] = p @ v, p @ v.abs()
    return out, lse, spread


def pool(g, n_pages, hkv, page, dtype, order="head", fill=None):
    """A pool of random pages (CPU) seen as [page][KV head][token][D], token-major if asked."""
    shape = (n_pages, hkv, page, D) if order == "head" else (n_pages, page, hkv, D)
    x = torch.randn(shape, generator=g) if fill is None else torch.full(shape, float(fill))
    x = x.to(dtype)
    return x if order == "head" else x.transpose(1, 2)


def to_cuda(x):
    """The same tensor on the GPU with the same strides."""
    if x.dim() == 4 and not x.is_contiguous():
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    return x.cuda()
