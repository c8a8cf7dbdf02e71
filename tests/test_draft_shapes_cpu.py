"""How the binding of the tree attention reads a queries' tensor that no q_tok_stride is given for: drafts
lie where its shape says, or the call is refused.  Without a GPU."""
import pytest

import paper_2608_14191_amd as P
from test_drafts_binding_cpu import _attention, _floats, calls, made                   # noqa: F401


def _stride(made, q, batch, max_draft, heads=4, **more):                              # noqa: F811
    _attention(q=q, batch=batch, max_draft=max_draft, n_q_heads=heads,
               out=_floats(batch, max_draft, heads, 128), **more)
    return made[-1][1][10]


def test_more_room_than_drafts(made):                                                 # noqa: F811
    """Contiguous buffers of more drafts a sequence than the call has: no one step leads through them."""
    for q in (_floats(3, 5, 4, 128), _floats(3, 5, 512), _floats(3, 5, 2, 2, 128), _floats(4, 3, 4, 128),
              _floats(4, 3, 1024)):
        n = len(made)
        with pytest.raises(P.AatcError) as e:
            _stride(made, q, 3, 2)
        assert e.value.status == 1 and len(made) == n, q.shape
    # one sequence has the first ones; one draft a sequence the first of each
    for q in (_floats(1, 5, 4, 128), _floats(5, 4, 128), _floats(1, 5, 512), _floats(5, 2, 2, 128)):
        assert _stride(made, q, 1, 2) == 512, q.shape
    assert _stride(made, _floats(3, 5, 4, 128), 3, 1) == 5 * 512
    # and with the step given the caller knows
    assert _stride(made, _floats(3, 5, 4, 128), 3, 2, q_tok_stride=512) == 512


def test_shapes_of_packed_drafts(made):                                               # noqa: F811
    """A contiguous tensor of just the numbers that are read is read in order, whatever its shape."""
    for q in (_floats(6, 4, 128), _floats(24, 128), _floats(6 * 512), _floats(3, 2, 4, 128), _floats(3, 2, 512),
              _floats(6, 2, 2, 128), _floats(3, 8, 128), _floats(1, 3, 2, 4, 128), _floats(3, 1, 4, 256),
              # more sequences, more tokens than are read
              _floats(9, 4, 128), _floats(5, 2, 4, 128), _floats(5, 2, 512), _floats(1, 5, 2, 4, 128),
              _floats(7 * 512 + 3), _floats(40, 128), _floats(9, 2, 2, 128)):
        assert _stride(made, q, 3, 2) == 512, q.shape
    for q in (_floats(3, 2, 128), _floats(6, 128), _floats(6, 1, 128), _floats(5, 2, 128), _floats(5, 2, 1, 128)):
        assert _stride(made, q, 3, 2, heads=1) == 128, q.shape


def test_more_heads_than_are_read(made):                                              # noqa: F811
    """A contiguous projection's output: the first heads of every token."""
    assert _stride(made, _floats(6, 8, 128), 3, 2) == 1024
    assert _stride(made, _floats(6, 1024), 3, 2) == 1024
    assert _stride(made, _floats(3, 2, 8, 128), 3, 2) == 1024
    assert _stride(made, _floats(3, 2, 1024), 3, 2) == 1024
    assert _stride(made, _floats(7, 5, 128), 3, 2) == 640
    with pytest.raises(P.AatcError):
        _stride(made, _floats(5, 8, 128), 3, 2)
