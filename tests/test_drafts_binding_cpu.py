"""What the bindings of drafted tokens and of sparse attention check before they call the library, without
a GPU: tensors that claim to be on a device, and the library's entry points replaced by a record."""
import pytest
import torch

import paper_2608_14191_amd as P
from paper_2608_14191_amd import _drafts, _paged, _sparse
from test_paged_binding_cpu import _cache, _floats, _i32, _on, _space, calls  # noqa: F401


@pytest.fixture
def made(calls, monkeypatch):                                                 # noqa: F811
    """(name, arguments) of every call that reaches the library."""
    got = []
    for module in (_drafts, _sparse):
        monkeypatch.setattr(module, "entry_point", lambda name: lambda *a: got.append((name, a)) or 0)
    return got


def _attention(**change):
    """Three sequences with two drafts each, four query heads over two KV heads."""
    a = dict(cache=_cache(), table=_i32(3, 5), seq_len=_i32(3), batch=3, max_draft=2, n_q_heads=4,
             q=_floats(6, 4, 128), softmax_scale=0.1, out=_floats(3, 2, 4, 128), workspace=_space())
    P.aatc_paged_tree_attention(**{**a, **change})


def _accept(**change):
    a = dict(cache=_cache(), table=_i32(3, 5), seq_len=_i32(3), batch=3, max_draft=2, drafted=_i32(3, 2),
             chosen=_i32(3, 2), path=_i32(3, 2), accepted=_i32(3), next=_i32(3), len_out=_i32(3))
    P.aatc_paged_tree_accept(**{**a, **change})


def _i8(*shape, where=0):
    return _on(torch.zeros(*shape, dtype=torch.int8), where)


def _bounds(**change):
    a = dict(cache=_cache(), table=_i32(3, 5), held=None, wanted=_i32(3), codes=_i8(4, 2, 2, 128),
             scales=_floats(4, 2))
    P.aatc_page_bounds(**{**a, **change})


def _sparse_attention(**change):
    a = dict(cache=_cache(), table=_i32(3, 5), seq_len=_i32(3), codes=_i8(4, 2, 2, 128),
             scales=_floats(4, 2), batch=3, n_q_heads=4, q=_floats(3, 4, 128), softmax_scale=0.1,
             picked=_i32(3, 2, 4), out=_floats(3, 4, 128), workspace=_space())
    P.aatc_paged_sparse_attention(**{**a, **change})


CALLS = {"aatc_paged_tree_attention": _attention, "aatc_paged_tree_accept": _accept,
         "aatc_page_bounds": _bounds, "aatc_paged_sparse_attention": _sparse_attention}
HALF = torch.zeros(64, dtype=torch.uint8)


def _refused(made, call, changes):
    call()
    n = len(made)
    for change in changes:
        with pytest.raises(P.AatcError) as e:
            call(**change)
        assert e.value.status == 1, change
    assert len(made) == n


@pytest.mark.parametrize("name", sorted(CALLS))
def test_page_tables(made, monkeypatch, name):
    """As a tensor and as a handle; on another device, of another type, or no table at all."""
    for table in (_i32(3, 5), P.PageTable(_i32(3, 5))):
        CALLS[name](table=table)
    assert [x for x, _ in made] == [name] * 2
    monkeypatch.setattr(_paged, "_device", lambda: 1)
    handle = P.PageTable(_i32(3, 5, where=1))
    monkeypatch.setattr(_paged, "_device", lambda: 0)
    _refused(made, CALLS[name], [dict(table=_i32(3, 5, where=1)), dict(table=handle),
                                 dict(table=_i32(3, 5).long())])


def test_buffers_of_tree_attention(made):
    _refused(made, _attention, [
        dict(seq_len=_i32(2)), dict(seq_len=_i32(3).long()), dict(seq_len=_i32(3, where=1)),
        dict(n_draft=_i32(2)), dict(n_draft=_i32(3, where=1)), dict(parent=_i32(3)), dict(parent=_i32(5)),
        dict(parent=_i32(6).float()), dict(out=_floats(3, 4, 128)), dict(out=_floats(3, 2, 4, 128).half()),
        dict(lse=_floats(23)), dict(lse=_floats(24).double()), dict(slopes=_floats(3)),
        dict(q=_floats(5, 4, 128)), dict(q=_floats(6, 4, 128), q_tok_stride=513),
        dict(workspace=_on(HALF[::2])), dict(workspace=_on(HALF[:1].expand(1 << 20)))])
    with pytest.raises(TypeError):
        _attention(q=_floats(6, 4, 128).double())
    _attention(n_draft=_i32(3), parent=_i32(3, 2), lse=_floats(3, 2, 4), slopes=_floats(4))


def test_strides_of_drafts(made):
    def stride_of(q, **more):
        _attention(q=q, **more)
        return made[-1][1][10]
    wide = _floats(6, 8, 128)
    assert stride_of(_floats(6, 4, 128)) == 512 and stride_of(_floats(24, 128)) == 512
    assert stride_of(_floats(3, 2, 4, 128)) == 512
    assert stride_of(wide[:, 4:]) == 1024 and stride_of(wide, q_tok_stride=1024) == 1024
    # sequences and drafts as two dimensions of a view; not where some of the drafts are left out
    assert stride_of(_floats(3, 2, 8, 128)[:, :, 4:]) == 1024
    assert stride_of(_floats(6, 1, 8, 128)[:, :, :4], max_draft=1, batch=3) == 1024
    assert stride_of(_floats(1, 6, 8, 128)[:, 1:3, :4], batch=1) == 1024
    _refused(made, _attention, [dict(q=_floats(3, 4, 4, 128)[:, :2]), dict(q=_floats(2, 3, 8, 128)[:, :, :4]),
                                dict(q=_floats(2, 2, 8, 128)[:, :, :4]), dict(q=wide[:5, :4]),
                                dict(q=_floats(4, 6, 128).transpose(0, 1)), dict(q=_floats(6, 4, 256)[..., ::2])])


def test_buffers_of_accept(made):
    lists = [dict(drafted=_i32(5)), dict(chosen=_i32(3)), dict(path=_i32(5)), dict(accepted=_i32(2)),
             dict(next=_i32(2)), dict(len_out=_i32(2)), dict(seq_len=_i32(2)), dict(n_draft=_i32(2)),
             dict(parent=_i32(5)), dict(path=_i32(3, 2).long()), dict(next=_i32(3, where=1)),
             dict(drafted=_on(torch.zeros(3, 4, dtype=torch.int32)[:, ::2]))]
    _refused(made, _accept, lists)


def test_layers_of_accept(made):
    """Every layer lies in the storage of the first one's tensors."""
    k, v = (torch.zeros(3, 4, 2, 16, 128) for _ in range(2))
    each = 4 * 2 * 16 * 128
    first = P.PagedCache(_on(k[0]), _on(v[0]))
    second = P.PagedCache(_on(k[1]), _on(v[1]))
    with_layers = lambda cache, n, stride: _accept(cache=cache, n_layers=n, layer_stride=stride)   # noqa: E731
    with_layers(first, 3, each)
    with_layers(second, 2, each)
    n = len(made)
    for bad in ((first, 4, each), (second, 3, each), (first, 3, each + 8), (first, 2, 0), (first, 2, -each)):
        with pytest.raises(P.AatcError):
            with_layers(*bad)
    assert len(made) == n


def test_buffers_of_bounds(made):
    _refused(made, _bounds, [
        dict(wanted=_i32(2)), dict(held=_i32(2)), dict(held=_i32(3).long()), dict(codes=_i8(3, 2, 2, 128)),
        dict(codes=_floats(4, 2, 2, 128)), dict(codes=_on(torch.zeros(4, 2, 2, 256, dtype=torch.int8)[..., ::2])),
        dict(codes=_i8(4, 2, 2, 128, where=1)), dict(scales=_floats(7)), dict(scales=_floats(4, 2).half()),
        dict(wanted=_i32(3, where=1))])


def test_buffers_of_sparse_attention(made):
    _refused(made, _sparse_attention, [
        dict(seq_len=_i32(2)), dict(codes=_i8(3, 2, 2, 128)), dict(scales=_floats(7)), dict(picked=_i32(3, 8)),
        dict(picked=_i32(2, 2, 4)), dict(picked=_i32(3, 1, 4)), dict(picked=_i32(3, 2, 4).long()),
        dict(picked=_on(torch.zeros(3, 2, 8, dtype=torch.int32)[..., ::2])), dict(out=_floats(2, 4, 128)),
        dict(lse=_floats(11)), dict(q=_floats(2, 4, 128)), dict(q=_floats(4, 3, 128).transpose(0, 1)),
        dict(workspace=_on(HALF[::2])), dict(picked=_i32(3, 2, 4, where=1))])
    _sparse_attention(q=_floats(3, 8, 128)[:, 4:], lse=_floats(3, 4))
    assert made[-1][1][9] == 1024
