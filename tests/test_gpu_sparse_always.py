"""aatc_paged_sparse_attention where the pages that are picked always fill all there is room for, so that
no score decides: a sink and the recent pages only."""
import pytest
import torch

from test_gpu_sparse import _case, _check, _run

pytestmark = pytest.mark.gpu


def _always(pages, first, last, most):
    """The picked list of a sequence of so many pages, all of them there."""
    some = list(range(pages)) if pages <= most else [*range(first), *range(pages - last, pages)]
    return some + [-1] * (most - len(some))


@pytest.mark.parametrize("first,last", [(4, 4), (1, 7), (7, 1), (8, 0), (0, 8)])
@pytest.mark.parametrize("batch,hkv", [(1, 1), (9, 4), (40, 8)])
def test_first_and_last_fill_the_room(first, last, batch, hkv):
    """Many rows in parts, some shorter than the room; the same lists and bits each time."""
    lens = [700 - 41 * (b % 17) for b in range(batch)]
    c = _case(60, lens, 2 * hkv, hkv, 16)
    picked, got = _check(c, 8, first, last)
    for b, n in enumerate(lens):
        want = _always(-(-n // 16), first, last, 8)
        assert all(picked[b, h].tolist() == want for h in range(hkv)), b
    for _ in range(3):
        again, same, _ = _run(c, 8, first, last)
        assert torch.equal(again, picked) and torch.equal(same, got)


@pytest.mark.parametrize("first,last,most", [(40, 24, 64), (64, 0, 64), (1500, 1000, 2500)])
def test_more_pages_than_in_registers(first, last, most):
    """9000 pages of a sequence: keys are read again for each pass; one list longer than LDS holds."""
    c = _case(61, [72000, 60], 2, 1, 8, "f16", "f16")
    picked, got = _check(c, most, first, last)
    assert picked[0, 0].tolist() == _always(9000, first, last, most)
    again, same, _ = _run(c, most, first, last)
    assert torch.equal(again, picked) and torch.equal(same, got)


def test_with_pages_that_are_not_there():
    """Room that missing pages leave: to the highest scores where there are more pages than room, all
    pages where there are not."""
    holes = [(0, 2, -1), (0, 30, 10 ** 6), (0, 43, -1)]
    holes += [(1, i, -1) for i in range(40) if i not in (0, 3, 17, 35)]
    holes += [(2, i, -1) for i in range(40) if i not in range(5, 13)]
    c = _case(62, [700, 640, 633], 8, 4, 16, holes=holes)
    picked, _ = _check(c, 8, 4, 4)
    assert all(x.tolist() == [0, 3, 17, 35] + [-1] * 4 for x in picked[1])
    assert all(x.tolist() == list(range(5, 13)) for x in picked[2])
    _check(c, 8, 0, 8)
    _check(c, 8, 8, 0)
