"""How the bindings of the attention of one token read a contiguous tensor of queries with more heads than
the call has, without a row stride given.  Without a GPU."""
import pytest

import paper_2608_14191_amd as P
from paper_2608_14191_amd import _paged
from test_drafts_binding_cpu import _floats, _sparse_attention, calls, made            # noqa: F401
from test_paged_binding_cpu import _cache, _i32, _joined, _space


def _decode_stride(made, q, batch, **more):                                           # noqa: F811
    P.aatc_paged_decode_attention(_cache(), _i32(3, 3), _i32(3), batch, 4, q, 0.1, _floats(3, 4, 128), _space(),
                                  **more)
    return made[-1][1][7]


def _sparse_stride(made, q, batch, **more):                                           # noqa: F811
    _sparse_attention(q=q, batch=batch, **more)
    return made[-1][1][9]


@pytest.mark.parametrize("stride_of", [_decode_stride, _sparse_stride])
def test_rows_of_contiguous_queries(made, monkeypatch, stride_of):                    # noqa: F811
    monkeypatch.setattr(_paged, "entry_point", lambda name: lambda *a: made.append((name, a)) or 0)
    # rows of more than the heads that are read: the first ones of each
    for q, step in ((_floats(3, 8, 128), 1024), (_floats(3, 1024), 1024), (_floats(5, 6, 128), 768),
                    (_floats(3, 2, 4, 128), 1024)):
        assert stride_of(made, q, 3) == step, q.shape
    # rows of just these, in any shape; one row; the caller's own step
    for q in (_floats(3, 4, 128), _floats(3, 2, 2, 128), _floats(3, 512), _floats(12, 128), _floats(1536),
              _floats(7, 4, 128), _floats(28, 128), _floats(4000), _floats(1, 5, 4, 128), _floats(1, 3, 4, 128)):
        assert stride_of(made, q, 3) == 512, q.shape
    assert stride_of(made, _floats(1, 8, 128), 1) == 512
    assert stride_of(made, _floats(3, 8, 128), 3, q_stride=512) == 512
    n = len(made)
    for q in (_floats(2, 4, 128), _floats(2, 5, 128)):
        with pytest.raises(P.AatcError):
            stride_of(made, q, 3)
    assert len(made) == n


def test_joined_attention_takes_packed_rows(calls):                                   # noqa: F811
    """Its C entry point has no row stride: rows of more heads are refused."""
    good = _joined()
    P.aatc_decode_attention_paged(**{**good, "q": _floats(3, 4, 128)})
    n = len(calls)
    for q in (_floats(2, 8, 128), _floats(2, 1024), _floats(3, 6, 128)):
        with pytest.raises(P.AatcError) as e:
            P.aatc_decode_attention_paged(**{**good, "q": q})
        assert e.value.status == 1
    assert len(calls) == n
