"""aatc_pages_reserve where entries behind the held tokens name pages already: reserved ahead, left by
a rollback, shared by a fork.  Against a plain sequential form, with the counts recounted."""
import pytest
import torch

import paper_2608_14191_amd as P

pytestmark = pytest.mark.gpu


def _counts(table, n_pages):
    t = table[(table >= 0) & (table < n_pages)].long()
    return torch.bincount(t, minlength=n_pages).int()


def _sequential(table, ref, page, held, wanted):
    """Row after row, entry after entry: what an entry's page lacks is a page, or one of its own."""
    rows, entries = table.shape
    n_pages, most = len(ref), entries * page
    before, table, ref = (table, ref), table.clone(), ref.clone()
    count = ref.clone()
    free = [i for i in range(n_pages) if ref[i] <= 0]
    taken, pairs = 0, torch.full((rows, 2), -1).int()
    for b in range(rows):
        lo, hi = (min(max(int(x[b]), 0), most) for x in (held, wanted))
        if hi <= lo:
            continue
        for e in range(lo // page, -(-hi // page)):
            begun = e == lo // page and lo % page != 0
            old = int(table[b, e])
            named = 0 <= old < n_pages and int(count[old]) > 0
            shared = named and int(ref[old]) > 1
            if not (shared or (not begun and not named)):
                continue
            if shared:
                ref[old] -= 1
            if taken < len(free):
                table[b, e] = free[taken]
                ref[free[taken]] = 1
                if begun:
                    pairs[b] = torch.tensor([old, free[taken]])
            taken += 1
    if taken > len(free):
        return (*before, torch.full((rows, 2), -1).int(), taken - len(free))
    return table, ref, pairs, 0


class _State:
    def __init__(self, rows, entries, n_pages, page):
        self.page, self.n_pages, self.rows = page, n_pages, rows
        self.table = torch.full((rows, entries), -1).int().cuda()
        self.ref = torch.zeros(n_pages).int().cuda()
        self.space = torch.empty(P.aatc_pages_workspace_bytes(rows, n_pages), dtype=torch.uint8, device="cuda")

    def reserve(self, held, wanted):
        """The call, compared with the sequential form: (pairs, lacking)."""
        held, wanted = (torch.as_tensor(x).int() for x in (held, wanted))
        want = _sequential(self.table.cpu(), self.ref.cpu(), self.page, held, wanted)
        pairs = torch.full((self.rows, 2), 99).int().cuda()
        lacking = torch.full((1,), 99).int().cuda()
        P.aatc_pages_reserve(self.table, self.ref, self.page, held.cuda(), wanted.cuda(), pairs, lacking,
                             self.space)
        assert int(lacking) == want[3]
        assert torch.equal(self.table.cpu(), want[0])
        assert torch.equal(self.ref.cpu(), want[1])
        assert torch.equal(pairs.cpu(), want[2])
        self.counted()
        return pairs.cpu(), want[3]

    def counted(self):
        assert torch.equal(self.ref.cpu(), _counts(self.table.cpu(), self.n_pages))


def test_reserved_ahead_and_forked():
    s = _State(2, 4, 10, 16)
    s.reserve([0, 0], [40, 0])
    P.aatc_pages_fork(s.table, s.table, s.ref, torch.tensor([[0, 1]]).int().cuda())
    pairs, _ = s.reserve([10, 10], [10, 40])             # the child writes: pages of its own
    assert pairs[1].tolist() == [0, 3]
    assert s.table.cpu().tolist() == [[0, 1, 2, -1], [3, 4, 5, -1]]
    pairs, _ = s.reserve([10, 40], [40, 40])             # the parent has its own by now
    assert torch.all(pairs == -1) and s.table.cpu()[0].tolist() == [0, 1, 2, -1]


def test_rolled_back_and_grown_again():
    s = _State(1, 6, 12, 8)
    s.reserve([0], [40])
    s.reserve([9], [33])                                 # back to 9 tokens: its pages are still there
    assert s.table.cpu()[0].tolist() == [0, 1, 2, 3, 4, -1]
    s.reserve([16], [48])
    assert s.table.cpu()[0].tolist() == [0, 1, 2, 3, 4, 5]
    P.aatc_pages_free(s.table, s.ref, torch.zeros(1).int().cuda())
    assert torch.all(s.ref == 0)


def test_the_same_call_twice():
    s = _State(3, 4, 12, 16)
    s.reserve([0, 0, 5], [33, 16, 20])
    once = s.table.cpu()
    s.reserve([0, 0, 5], [33, 16, 20])
    assert torch.equal(s.table.cpu(), once)


def test_all_holders_grow():
    """Rows that share pages ahead all get their own but the last, which keeps them."""
    s = _State(5, 3, 40, 8)
    s.reserve([0] * 5, [24, 0, 0, 0, 0])
    P.aatc_pages_fork(s.table, s.table, s.ref, torch.tensor([[0, i] for i in range(1, 5)]).int().cuda())
    pairs, _ = s.reserve([4] * 5, [24] * 5)
    assert s.table.cpu()[4].tolist() == [0, 1, 2] and pairs[4].tolist() == [-1, -1]
    assert torch.all(s.ref.cpu()[:15] == 1)


def test_entries_that_name_free_or_no_pages():
    """A page of count 0, and entries outside the pool, are no pages to keep."""
    s = _State(2, 4, 8, 8)
    s.table.copy_(torch.tensor([[7, 8, -5, 2 ** 31 - 1], [1, 1, -1, -1]]).int())
    s.ref[1] = 2
    held, wanted = torch.tensor([0, 0]).int(), torch.tensor([32, 0]).int()
    want = _sequential(s.table.cpu(), s.ref.cpu(), 8, held, wanted)
    pairs, lacking = torch.zeros(2, 2).int().cuda(), torch.zeros(1).int().cuda()
    P.aatc_pages_reserve(s.table, s.ref, 8, held.cuda(), wanted.cuda(), pairs, lacking, s.space)
    assert s.table.cpu()[0].tolist() == [0, 2, 3, 4]
    assert torch.equal(s.table.cpu(), want[0]) and torch.equal(s.ref.cpu(), want[1])


def test_too_few_pages_for_copies_ahead():
    s = _State(2, 3, 5, 8)
    s.reserve([0, 0], [24, 0])
    P.aatc_pages_fork(s.table, s.table, s.ref, torch.tensor([[0, 1]]).int().cuda())
    before = s.table.cpu(), s.ref.cpu()
    _, lacking = s.reserve([3, 3], [3, 24])              # three pages of its own, two free
    assert lacking == 1
    assert torch.equal(s.table.cpu(), before[0]) and torch.equal(s.ref.cpu(), before[1])


# Calls of one claim a row, of more claims than the workgroup has threads, of more rows than that.
@pytest.mark.parametrize("rows,entries,n_pages,page", [(1, 6000, 9000, 8), (6, 40, 300, 16), (70, 30, 3000, 8),
                                                       (3, 900, 6000, 64), (1500, 5, 9000, 8), (2100, 3, 3500, 16),
                                                       (7, 4000, 30000, 8)])
@pytest.mark.parametrize("seed", [0, 1])
def test_random_histories(rows, entries, n_pages, page, seed):
    g = torch.Generator().manual_seed(seed + rows)
    s = _State(rows, entries, n_pages, page)
    most = entries * page
    draw = lambda hi: torch.randint(0, hi, (rows,), generator=g)                    # noqa: E731
    held = torch.zeros(rows).long()
    for step in range(4):
        ahead = held + torch.where(draw(3) > 0, draw(max(2, 2 * most // 5)), torch.zeros(rows).long())
        _, lacking = s.reserve(held, ahead)
        if not lacking:                                  # some of what was made room for is used
            held = held + (torch.rand(rows, generator=g) * (ahead.clamp(max=most) - held).clamp(min=0)).long()
        if rows > 1:                                     # forks, ahead of the tokens too
            perm = torch.randperm(rows, generator=g)
            n = max(1, rows // 3)
            src, dst = perm[torch.randint(0, rows - n, (n,), generator=g)], perm[rows - n:]
            P.aatc_pages_free(s.table, s.ref, dst.int().cuda())
            P.aatc_pages_fork(s.table, s.table, s.ref, torch.stack([src, dst], 1).int().cuda())
            held[dst] = held[src]
        held = torch.where(draw(4) == 0, held // 2, held)    # rolled back
        s.counted()
