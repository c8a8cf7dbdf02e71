"""What the binding of the paged calls checks before it calls the library, without a GPU: tensors that
claim to be on a device, and the library's entry points replaced by a record of their calls."""
import pytest
import torch

import paper_2608_14191_amd as P
from paper_2608_14191_amd import _paged
from test_paged_cpu import A, TABLE, UNSUPPORTED, _call


class _On(torch.Tensor):
    """A CPU tensor that says it is on GPU `where`."""

    where = 0

    def get_device(self):
        return self.where


def _on(t, where=0):
    t = t.as_subclass(_On)
    t.where = where
    return t


@pytest.fixture
def calls(monkeypatch):
    made = []
    _paged._torch()
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(_paged, "_device", lambda: 0)
    monkeypatch.setattr(_paged, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(_paged, "entry_point", lambda name: lambda *a: made.append(name) or 0)
    return made


def _i32(*shape, where=0):
    return _on(torch.zeros(*shape, dtype=torch.int32), where)


def _cache(pages=4, heads=2, page=16):
    return P.PagedCache(*(_on(torch.zeros(pages, heads, page, 128)) for _ in range(2)))


def _floats(*shape):
    return _on(torch.zeros(*shape))


def _space():
    return _on(torch.zeros(64, dtype=torch.uint8))


def _calls_with(table):
    """Every call that takes a page table, with `table` in its place."""
    x, good = _floats(1, 2, 128), _i32(2, 3)
    return {
        "aatc_paged_append": lambda: P.aatc_paged_append(_cache(), table, 1, x, x, 256, 256, None, _i32(1)),
        "aatc_paged_decode_attention": lambda: P.aatc_paged_decode_attention(
            _cache(), table, _i32(1), 1, 2, x, 0.1, _floats(1, 2, 128), _space()),
        "aatc_decode_attention_paged": lambda: P.aatc_decode_attention_paged(**{**_joined(), "table": table}),
        "aatc_pages_fork": lambda: P.aatc_pages_fork(table, good, _i32(4), _i32(1, 2)),
        "aatc_pages_fork ": lambda: P.aatc_pages_fork(good, table, _i32(4), _i32(1, 2)),
        "aatc_pages_free": lambda: P.aatc_pages_free(table, _i32(4), _i32(1)),
        "aatc_pages_reserve": lambda: P.aatc_pages_reserve(table, _i32(4), 16, _i32(2), _i32(2), _i32(2, 2),
                                                           _i32(1), _space()),
        "aatc_pages_compact": lambda: P.aatc_pages_compact(table, _i32(4), good, _i32(4), _i32(2, 2), _i32(1),
                                                           _space()),
        "aatc_pages_compact ": lambda: P.aatc_pages_compact(good, _i32(4), table, _i32(4), _i32(2, 2), _i32(1),
                                                            _space()),
    }


def _joined():
    """Arguments of the joined attention: two sequences, two KV heads, 64 tokens, 44-byte records."""
    u8 = lambda *s: _on(torch.zeros(*s, dtype=torch.uint8))                      # noqa: E731
    alpha = lambda: _on(torch.zeros(2, 2, 64, dtype=torch.int16))               # noqa: E731
    params = P.library().aatc_params_bytes(2)
    return dict(dev_params_k=u8(params), dev_params_v=u8(params), batch=2, n_q_heads=4, n_kv_heads=2,
                q=_floats(2, 4, 128), k_codes=u8(2, 2, 64, 44), k_alpha=alpha(), v_codes=u8(2, 2, 1, 64 * 44),
                v_alpha=alpha(), seq_len=_i32(2), cap=64, k_record_bytes=44, v_record_bytes=44,
                softmax_scale=0.1, cache=_cache(), table=_i32(2, 3), page_len=_i32(2),
                out=_floats(2, 4, 128), workspace=_space())


@pytest.mark.parametrize("name", sorted(_calls_with(None)))
def test_page_tables_on_another_device(calls, monkeypatch, name):
    """As a tensor and as a handle, which may have been made while its device was the current one."""
    for table in (_i32(2, 3), P.PageTable(_i32(2, 3))):
        _calls_with(table)[name]()
    assert calls == [name.strip()] * 2
    monkeypatch.setattr(_paged, "_device", lambda: 1)
    handle = P.PageTable(_i32(2, 3, where=1))
    monkeypatch.setattr(_paged, "_device", lambda: 0)
    for table in (_i32(2, 3, where=1), handle):
        with pytest.raises(P.AatcError) as e:
            _calls_with(table)[name]()
        assert e.value.status == 1 and "device" in str(e.value)
    assert len(calls) == 2


def test_joined_attention_buffers(calls):
    """Types and sizes of what the call reads: codes, scales, parameters and queries."""
    good = _joined()
    P.aatc_decode_attention_paged(**good)
    P.aatc_decode_attention_paged(**{**good, "k_alpha": good["k_alpha"].view(torch.float16)})
    assert len(calls) == 2
    u8 = lambda *s: _on(torch.zeros(*s, dtype=torch.uint8))                      # noqa: E731
    params = good["dev_params_k"].numel()
    bad = [dict(dev_params_k=u8(params - 1)), dict(dev_params_v=u8(params - 1)), dict(k_codes=u8(2, 2, 63, 44)),
           dict(v_codes=u8(1, 2, 1, 64 * 44)), dict(k_codes=_on(torch.zeros(2, 2, 64, 88, dtype=torch.uint8)[..., ::2], 0)),
           dict(k_record_bytes=48), dict(v_record_bytes=48), dict(cap=128), dict(k_alpha=_floats(2, 2, 64)),
           dict(v_alpha=_on(torch.zeros(2, 2, 63, dtype=torch.int16))), dict(k_alpha=u8(2, 2, 128)),
           dict(q=_floats(1, 4, 128)), dict(q=_floats(2, 6, 128)[:, :4]), dict(q=_floats(4, 2, 128).transpose(0, 1)),
           dict(k_codes=_on(torch.zeros(2, 2, 64, 44, dtype=torch.uint8), 1)), dict(seq_len=_i32(1)),
           dict(page_len=_i32(2).long()), dict(out=_floats(2, 3, 128))]
    for change in bad:
        with pytest.raises(P.AatcError) as e:
            P.aatc_decode_attention_paged(**{**good, **change})
        assert e.value.status == 1, change
    assert len(calls) == 2


def test_lists_of_pairs(calls):
    """[n][2], or nothing at all: rows of other lengths would be read as other pairs."""
    pools = _on(torch.zeros(1, 4, 8, dtype=torch.int32))
    fork = lambda pairs: P.aatc_pages_fork(_i32(4, 3), _i32(4, 3), _i32(9), pairs)       # noqa: E731
    copy = lambda pairs: P.aatc_pages_copy(pools, pairs)                                  # noqa: E731
    for call in (fork, copy):
        call(_i32(3, 2))
        call(_i32(0, 2))
        call(_i32(0))
        made = len(calls)
        for bad in (_i32(3, 3), _i32(3, 4), _i32(3, 2, 2), _i32(6), _i32(3, 1), _i32(3, 2).long(),
                    _on(torch.zeros(3, 4, dtype=torch.int32)[:, ::2])):
            with pytest.raises(P.AatcError):
                call(bad)
        assert len(calls) == made


def test_rows_of_queries(monkeypatch, calls):
    """Without q_stride rows lie as the tensor has them, the heads of a wider projection too."""
    got = []
    monkeypatch.setattr(_paged, "entry_point", lambda name: lambda *a: got.append(a[7]) or 0)

    def stride_of(q, batch, **more):
        P.aatc_paged_decode_attention(_cache(), _i32(3, 3), _i32(3), batch, 4, q, 0.1, _floats(3, 4, 128),
                                      _space(), **more)
        return got[-1]
    wide = _floats(3, 8, 128)
    assert stride_of(_floats(3, 4, 128), 3) == 512
    assert stride_of(_floats(12, 128), 3) == 512
    assert stride_of(_floats(4 * 3 * 128), 3) == 512
    assert stride_of(wide[:, :4], 3) == 1024 and stride_of(wide[:, 4:], 3) == 1024
    assert stride_of(wide.reshape(3, 1024)[:, 512:], 3) == 1024
    assert stride_of(wide[:, 4:], 1) == 512                 # (one row: any)
    assert stride_of(wide[:, 4:], 3, q_stride=1024) == 1024
    assert stride_of(wide, 3, q_stride=1024) == 1024
    for bad in (_floats(4, 3, 128).transpose(0, 1), _floats(3, 4, 256)[..., ::2], wide[:2, :4]):
        made = len(got)
        with pytest.raises(P.AatcError):
            stride_of(bad, 3)
        assert len(got) == made


def test_workspaces_are_contiguous(calls):
    """(An expanded tensor has more elements than memory.)"""
    for bad in (_on(torch.zeros(1, dtype=torch.uint8).expand(1 << 20)), _on(torch.zeros(64, dtype=torch.uint8)[::2])):
        with pytest.raises(P.AatcError):
            P.aatc_paged_decode_attention(_cache(), _i32(3, 3), _i32(3), 3, 4, _floats(3, 4, 128), 0.1,
                                          _floats(3, 4, 128), bad)
        with pytest.raises(P.AatcError):
            P.aatc_decode_attention_paged(**{**_joined(), "workspace": bad})
        with pytest.raises(P.AatcError):
            P.aatc_pages_reserve(_i32(2, 3), _i32(4), 16, _i32(2), _i32(2), _i32(2, 2), _i32(1), bad)
        with pytest.raises(P.AatcError):
            P.aatc_pages_compact(_i32(2, 3), _i32(4), _i32(2, 3), _i32(4), _i32(2, 2), _i32(1), bad)
    assert calls == []


def test_forks_of_one_call():
    """The work grows with the square of the pairs: 2^18 at most (2^24 would take minutes)."""
    fork = dict(src=(P.PageTable, TABLE), dst=(P.PageTable, TABLE), ref=A, n_pages=100, pairs=A, n=0, stream=None)
    for n in ((1 << 18) + 1, 1 << 20, (1 << 24) - 1, 1 << 24):
        assert _call("aatc_pages_fork", fork, n=n) == UNSUPPORTED
