"""Attention over pages with scores of 2^20 and more, whose last bit is worth many powers of two of a
weight: equal scores have equal weights, lower ones none, and nothing overflows."""
import pytest
import torch

import paper_2608_14191_amd as P
import test_gpu_sparse as sparse
from drafts_ref import page_bounds, tree_attention
from paged_ref import TYPES, to_cuda
from test_gpu_tree_attention import D, SCALE, _case, _check, _close, _run
from test_gpu_tree_large import _slots

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,qtype,powers", [("bf16", "bf16", (20, 22, 25, 29, 33, 60, 100)),
                                                ("f32", "f32", (20, 22, 25, 29, 33, 60, 100)),
                                                ("f16", "f16", (20, 22, 24, 25, 26, 27)),
                                                ("f16", "f32", (20, 22, 24, 25, 26, 27)),
                                                ("bf16", "f32", (22, 33, 100))])
@pytest.mark.parametrize("drafts", [3, 20, 64])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores(cache, qtype, powers, drafts, sign):
    """Scores of +-2^20 and more: the two tokens with the highest one share the weight, all others have
    none.  (A score's last bit is then worth many powers of two of its weight.)"""
    for power in powers:
        c = _case(41, [300, 90], drafts, 4, 2, 16, cache, qtype, tree="chain")
        half = power // 2 + 2                          # (both factors fit float16)
        for b, m in enumerate(c["lens"].tolist()):
            pages, slot = _slots(c, b, m + drafts)
            low = 0.5 if sign > 0 else 1.75
            c["k"][pages, :, slot] = 0
            c["k"][pages, :, slot, 0] = low * 2.0 ** half * sign
            for t in (5, m // 2 + 33):
                p, s = c["table"][b, t // 16].long(), t % 16
                c["k"][p, :, s, 0] = 1.1328125 * 2.0 ** half * sign
        c["q"][:] = 0
        c["q"][..., 0] = 1.2890625 * 2.0 ** (power - half + 3)
        got = _check(c)
        assert torch.isfinite(got).all()
        for b, m in enumerate(c["lens"].tolist()):
            two = [c["v"][c["table"][b, t // 16].long(), :, t % 16].double() for t in (5, m // 2 + 33)]
            want = ((two[0] + two[1]) / 2).repeat_interleave(2, 0)
            assert (got[b].double() - want).norm() <= 1e-6 * got[b].double().norm(), power


def test_scores_that_rise_to_large_ones():
    """Small scores first, then larger and larger ones, tile by tile: the largest decides."""
    for cache in ("bf16", "f16", "f32"):
        c = _case(42, [320], 6, 4, 2, 16, cache, cache, tree="chain")
        pages, slot = _slots(c, 0, 326)
        c["k"][pages, :, slot] = 0
        steps = 2.0 ** torch.arange(326).div(22, rounding_mode="floor")
        c["k"][pages, :, slot, 0] = steps[:, None].to(TYPES[cache])
        c["q"][:] = 0
        c["q"][..., 0] = 1.1328125 * 2.0 ** 13
        got, lse = _run(c)
        want, want_lse, spread = tree_attention(c["k"], c["v"], c["table"], c["lens"], c["q"], SCALE, None, None)
        _close(got, lse, want, want_lse, spread)


def _large_keys(c, power, cache, qtype):
    """Two tokens of each sequence with the highest score, 2^power and more, all others with half of it;
    returns what the heads end as: the mean of the two tokens' values."""
    half = power // 2 + 2
    want = []
    for b, m in enumerate(c["lens"].tolist()):
        pages, slot = _slots(c, b, m)
        c["k"][pages, :, slot] = 0
        c["k"][pages, :, slot, 0] = 0.5 * 2.0 ** half
        two = []
        for t in (5, m // 2 + 33):
            p, s = c["table"][b, t // 16].long(), t % 16
            c["k"][p, :, s, 0] = 1.1328125 * 2.0 ** half
            two.append(c["v"][p, :, s].double())
        want.append(((two[0] + two[1]) / 2).repeat_interleave(2, 0))
    c["q"][:] = 0
    c["q"][..., 0] = 1.2890625 * 2.0 ** (power - half + 3)
    return torch.stack(want)


TYPES_AND_POWERS = [("bf16", "bf16", (20, 25, 33, 60, 100)), ("f32", "f32", (20, 25, 33, 60, 100)),
                    ("f16", "f16", (20, 22, 24, 25, 26, 27)), ("f16", "f32", (20, 22, 24, 25, 26, 27))]


@pytest.mark.parametrize("cache,qtype,powers", TYPES_AND_POWERS)
def test_large_scores_of_one_token(cache, qtype, powers):
    for power in powers:
        c = sparse._case(44, [300, 90, 2000], 4, 2, 16, cache, qtype)
        want = _large_keys(c, power, cache, qtype)
        out = torch.empty(3, 4, D, device="cuda")
        ws = torch.zeros(P.aatc_paged_decode_workspace_bytes(3, 4, 2), dtype=torch.uint8, device="cuda")
        P.aatc_paged_decode_attention(P.PagedCache(to_cuda(c["k"]), to_cuda(c["v"])), c["table"].cuda(),
                                      c["lens"].cuda(), 3, 4, c["q"].cuda(), SCALE, out, ws)
        assert (out.cpu().double() - want).norm() <= 1e-6 * want.norm(), power


@pytest.mark.parametrize("cache,qtype,powers", TYPES_AND_POWERS)
def test_large_scores_of_picked_pages(cache, qtype, powers):
    for power in powers:
        c = sparse._case(45, [300, 90, 2000], 4, 2, 16, cache, qtype)
        want = _large_keys(c, power, cache, qtype)
        for b, m in enumerate(c["lens"].tolist()):
            for i in range(-(-m // 16)):
                at = int(c["table"][b, i])
                for h in range(2):
                    c["codes"][at, h], c["scales"][at, h] = page_bounds(c["k"][at, h, :min(16, m - 16 * i)])
        for most in (12, 200):
            picked, got = sparse._check(c, most)
            assert (got.double() - want).norm() <= 1e-6 * want.norm(), power
