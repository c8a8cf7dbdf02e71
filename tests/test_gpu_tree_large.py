"""aatc_paged_tree_attention with values near the end of float32's range: finite where one token's attention
is."""
import pytest
import torch

import paper_2608_14191_amd as P
from paged_ref import TYPES, to_cuda
from test_gpu_tree_attention import D, SCALE, _case, _check

pytestmark = pytest.mark.gpu


def _slots(c, b, n):
    """(pages, slots) of the first n tokens of sequence b."""
    t = torch.arange(n)
    page = c["k"].shape[2]
    return c["table"][b].long()[t // page], t % page


def _one_by_one(c, drafts):
    """aatc_paged_decode_attention of each draft of a chain."""
    batch, _, hq, _ = c["q"].shape
    hkv = c["k"].shape[1]
    cache = P.PagedCache(to_cuda(c["k"]), to_cuda(c["v"]))
    ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(batch, hq, hkv), dtype=torch.uint8, device="cuda")
    out = torch.zeros(drafts, batch, hq, D, device="cuda")
    for i in range(drafts):
        P.aatc_paged_decode_attention(cache, c["table"].cuda(), (c["lens"] + i + 1).cuda(), batch, hq,
                                      c["q"][:, i].contiguous().cuda(), SCALE, out[i], ws)
    return out.transpose(0, 1).cpu()


@pytest.mark.parametrize("cache,qtype", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("drafts", [3, 20, 64])
@pytest.mark.parametrize("n", [200, 5000])
def test_large_values(cache, qtype, drafts, n):
    """Values near 2^128 / n under scores that rise by 2^7: weights of at most 1 keep the sums finite.

    Scores rise along the sequence from 0 to 7.2 (exponents of 2), so the weights relative to the largest
    sum to n / (7.2 ln 2) = n / 5, and values of at most 2^127 / n to a quarter of float32's range."""
    c = _case(40, [n, n // 3], drafts, 4, 2, 16, cache, qtype, tree="chain")
    top = 2.0 ** 126 / n
    g = torch.Generator().manual_seed(1)
    for b, m in enumerate(c["lens"].tolist()):
        pages, slot = _slots(c, b, m + drafts)
        c["k"][pages, :, slot] = 0
        c["k"][pages, :, slot, 0] = (5 / 8 / SCALE * torch.arange(m + drafts) / (m + drafts))[:, None].to(TYPES[cache])
        c["v"][pages, :, slot] = (top * (1 + torch.rand(m + drafts, 2, D, generator=g))).to(TYPES[cache])
    c["q"][..., 0] = 8
    got = _check(c)
    assert torch.isfinite(got).all()
    if drafts == 3:
        one = _one_by_one(c, drafts)
        assert (one.double() - got.double()).norm() <= 4e-6 * got.double().norm()


@pytest.mark.parametrize("cache,qtype", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("drafts", [3, 20, 64])
def test_large_values_behind_low_scores(cache, qtype, drafts):
    """Every wave's first tile scores 7.2 less (exponents of 2) than all later ones: 2^7.2 times as many of
    their values of 2^117 or more as one tile has tokens would pass 2^128; weighted by 1 they do not."""
    n, low = (500, 256) if cache == "bf16" else (250, 128)
    c = _case(43, [n, n - 9], drafts, 4, 2, 16, cache, qtype, tree="chain")
    g = torch.Generator().manual_seed(2)
    for b, m in enumerate(c["lens"].tolist()):
        pages, slot = _slots(c, b, m + drafts)
        c["k"][pages, :, slot] = 0
        c["k"][pages[low:], :, slot[low:], 0] = 5 / 8 / SCALE
        c["v"][pages, :, slot] = (2.0 ** 126 / n * (1 + torch.rand(m + drafts, 2, D, generator=g))).to(TYPES[cache])
    c["q"][..., 0] = 8
    assert torch.isfinite(_check(c)).all()
