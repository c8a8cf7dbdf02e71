"""Page tables on the device against a plain sequential form: fork, free, reserve (with copies on
write), compact and copy."""
import pytest
import torch

import paper_2608_14191_amd as P

pytestmark = pytest.mark.gpu


def _counts(table, n_pages):
    t = table[(table >= 0) & (table < n_pages)].long()
    return torch.bincount(t, minlength=n_pages).int()


def _space(rows, n_pages):
    return torch.empty(P.aatc_pages_workspace_bytes(rows, n_pages), dtype=torch.uint8, device="cuda")


def _random(seed, rows, entries, n_pages, used=0.6):
    g = torch.Generator().manual_seed(seed)
    table = torch.randint(0, n_pages, (rows, entries), generator=g).int()
    table[torch.rand(rows, entries, generator=g) > used] = -1
    return g, table, _counts(table, n_pages)


@pytest.mark.parametrize("rows,entries,n_pages,n", [(4, 3, 10, 2), (64, 50, 500, 30),
                                                    (300, 1, 40, 150), (8, 1000, 3000, 4)])
def test_fork_and_free(rows, entries, n_pages, n):
    g, table, ref = _random(rows, rows, entries, n_pages)
    perm = torch.randperm(rows, generator=g)
    src = perm[torch.randint(0, rows - n, (n,), generator=g)]
    dst = perm[rows - n:]
    pairs = torch.stack([src, dst], 1).int()
    extra = torch.tensor([[int(src[0]), int(dst[0])], [-1, int(dst[0])], [rows, 0], [0, rows],
                          [0, -1]]).int()
    pairs = torch.cat([torch.stack([perm[:1], dst[:1]], 1).int(), pairs, extra])   # dst[0]: twice, last wins
    t, r = table.cuda(), ref.cuda()
    other = torch.full((rows, entries + 5), -7, dtype=torch.int32).cuda()
    P.aatc_pages_fork(t, t, r, pairs.cuda())
    want, count = table.clone(), ref.clone()
    for a, b in zip(src.tolist(), dst.tolist()):
        want[b] = table[a]
        count += _counts(table[a], n_pages)
    assert torch.equal(t.cpu(), want) and torch.equal(r.cpu(), count)
    # into another table of padded rows
    P.aatc_pages_fork(t, other[:, :entries], r, torch.tensor([[1, 2]]).int().cuda())
    assert torch.equal(other.cpu()[2, :entries], want[1]) and torch.all(other[:, entries:] == -7)
    count += _counts(want[1], n_pages)
    # free: rows listed twice, rows that do not exist
    rows_off = torch.tensor([0, 1, 1, rows - 1, -1, rows, 0]).int()
    P.aatc_pages_free(t, r, rows_off.cuda())
    for b in {0, 1, rows - 1}:
        count -= _counts(want[b], n_pages)
        want[b] = -1
    assert torch.equal(t.cpu(), want) and torch.equal(r.cpu(), count)


def _reserve(table, ref, page, held, wanted):
    """The sequential form."""
    rows, entries = table.shape
    n_pages, most = len(ref), entries * page
    before, table, ref = (table, ref), table.clone(), ref.clone()
    free = [i for i in range(n_pages) if ref[i] <= 0]
    taken, pairs = 0, torch.full((rows, 2), -1).int()
    for b in range(rows):
        lo, hi = (min(max(int(x[b]), 0), most) for x in (held, wanted))
        if hi <= lo:
            continue
        places = list(range(-(-lo // page), -(-hi // page)))
        if lo % page:
            old = int(table[b, lo // page])
            if 0 <= old < n_pages and ref[old] > 1:
                ref[old] -= 1
                if taken < len(free):
                    pairs[b] = torch.tensor([old, free[taken]])
                places.insert(0, lo // page)
        for i in places:
            if taken < len(free):
                table[b, i] = free[taken]
                ref[free[taken]] = 1
            taken += 1
    if taken > len(free):
        return (*before, torch.full((rows, 2), -1).int(), taken - len(free))
    return table, ref, pairs, 0


@pytest.mark.parametrize("rows,n_pages,page,grow", [(1, 8, 8, 1), (5, 64, 16, 1), (40, 900, 16, 40),
                                                    (40, 300, 8, 3), (1500, 40000, 8, 2),
                                                    (3, 20, 8, 400), (2500, 30000, 16, 1)])
@pytest.mark.parametrize("shared", [False, True])
def test_reserve(rows, n_pages, page, grow, shared):
    g = torch.Generator().manual_seed(rows + n_pages)
    entries = 8
    table = torch.full((rows, entries), -1).int()
    held = torch.randint(0, 4 * page, (rows,), generator=g).int()
    perm, at = torch.randperm(n_pages, generator=g).int(), 0
    for b in range(rows):
        if shared and b and torch.rand(1, generator=g) < 0.6:      # as a fork of an earlier row
            a = int(torch.randint(max(0, b - 4), b, (1,), generator=g))
            table[b], held[b] = table[a], held[a]
            continue
        need = -(-int(held[b]) // page)
        if at + need > n_pages * 3 // 4:
            held[b] = need = 0
        table[b, :need] = perm[at:at + need]
        at += need
    ref = _counts(table, n_pages)
    wanted = held + torch.randint(-1, grow + 1, (rows,), generator=g).int()
    want = _reserve(table, ref, page, held, wanted)
    t, r = table.cuda(), ref.cuda()
    pairs = torch.full((rows, 2), 99).int().cuda()
    lacking = torch.full((1,), 99).int().cuda()
    P.aatc_pages_reserve(t, r, page, held.cuda(), wanted.cuda(), pairs, lacking, _space(rows, n_pages))
    assert int(lacking) == want[3]
    assert torch.equal(t.cpu(), want[0]) and torch.equal(r.cpu(), want[1])
    assert torch.equal(pairs.cpu(), want[2])
    if not want[3]:
        assert torch.equal(r.cpu(), _counts(t.cpu(), n_pages))


def test_reserve_that_lacks_pages_changes_nothing():
    table = torch.tensor([[0, -1, -1], [0, -1, -1], [1, -1, -1]]).int()
    ref = torch.tensor([2, 1, 0]).int()
    t, r = table.cuda(), ref.cuda()
    pairs, lacking = torch.zeros(3, 2).int().cuda(), torch.zeros(1).int().cuda()
    held, wanted = torch.tensor([5, 5, 8]).int().cuda(), torch.tensor([6, 17, 24]).int().cuda()
    P.aatc_pages_reserve(t, r, 8, held, wanted, pairs, lacking, _space(3, 3))
    # one copy (the last holder of page 0 keeps it) and 0 + 2 + 2 pages, one free
    assert int(lacking) == 4
    assert torch.equal(t.cpu(), table) and torch.equal(r.cpu(), ref) and torch.all(pairs == -1)


@pytest.mark.parametrize("n_pages,rows,entries,used", [(1, 1, 1, 0.5), (2, 1, 2, 0.5), (7, 2, 3, 0.9),
                                                       (1000, 20, 20, 0.5), (40000, 64, 300, 0.8),
                                                       (5000, 3, 10, 0.0), (64, 64, 20, 1.0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(n_pages, rows, entries, used, in_place):
    g, table, ref = _random(n_pages, rows, entries, n_pages, used)
    if n_pages > 2:
        ref[n_pages - 1] += 1                        # named by another table
    live = [i for i in range(n_pages) if ref[i] > 0]
    n_live = len(live)
    holes = [i for i in range(n_live) if ref[i] <= 0]
    move = dict(zip([i for i in live if i >= n_live], holes))
    t, r = table.cuda(), ref.cuda()
    t_out, r_out = (t, r) if in_place else (torch.full_like(t, 77), torch.full_like(r, 77))
    pairs = torch.full((max(1, n_pages // 2), 2), 99).int().cuda()
    moves = torch.zeros(1).int().cuda()
    pools = torch.randint(-9, 9, (3, n_pages, 8), generator=g).int()
    dev = pools.cuda()
    P.aatc_pages_compact(t, r, t_out, r_out, pairs, moves, _space(rows, n_pages))
    P.aatc_pages_copy(dev, pairs, n_pairs=moves)
    assert int(moves) == len(move)
    want = torch.full((n_pages // 2, 2), -1).int()
    if move:
        want[:len(move)] = torch.tensor(sorted(move.items())).int()
    assert torch.equal(pairs.cpu()[:n_pages // 2], want)
    to = torch.arange(n_pages).int()
    new_ref = torch.where(torch.arange(n_pages) < n_live, ref, torch.zeros_like(ref))
    for a, b in move.items():
        to[a], new_ref[b] = b, ref[a]
        pools[:, b] = pools[:, a]
    assert torch.equal(t_out.cpu(), torch.where(table >= 0, to[table.clamp(min=0).long()], table))
    assert torch.equal(r_out.cpu(), new_ref)
    assert torch.equal(dev.cpu(), pools)


@pytest.mark.parametrize("page_bytes", [16, 48, 4096, 16384 + 16, 100000 * 16])
@pytest.mark.parametrize("n_pools", [1, 3])
def test_copy(page_bytes, n_pools):
    n_pages = 12
    g = torch.Generator().manual_seed(page_bytes)
    pools = torch.randint(-2 ** 31, 2 ** 31 - 1, (n_pools, n_pages, page_bytes // 4), generator=g,
                          dtype=torch.int64).int()
    pairs = torch.tensor([[0, 5], [3, 4], [-1, 6], [2, 12], [12, 7], [8, -1], [9, 9], [0, 10]]).int()
    dev = pools.cuda()
    P.aatc_pages_copy(dev, pairs.cuda())
    want = pools.clone()
    want[:, 5], want[:, 4], want[:, 10] = pools[:, 0], pools[:, 3], pools[:, 0]
    assert torch.equal(dev.cpu(), want)
    for count, upto in ((0, 0), (1, 1), (-3, 0), (100, 8)):
        dev = pools.cuda()
        P.aatc_pages_copy(dev, pairs.cuda(), n_pairs=torch.tensor([count]).int().cuda())
        want = pools.clone()
        for a, b in pairs[:upto].tolist():
            if 0 <= a < n_pages and 0 <= b < n_pages:
                want[:, b] = pools[:, a]
        assert torch.equal(dev.cpu(), want)


def test_copy_of_a_part_of_the_pools():
    pools = torch.arange(4 * 6 * 4).reshape(4, 6, 4).int()
    dev = pools.cuda()
    P.aatc_pages_copy(dev[::2], torch.tensor([[1, 2]]).int().cuda())
    want = pools.clone()
    want[::2, 2] = want[::2, 1]
    assert torch.equal(dev.cpu(), want)
    P.aatc_pages_copy(dev, torch.zeros(0, 2).int().cuda())
    assert torch.equal(dev.cpu(), want)
