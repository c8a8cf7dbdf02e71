"""The paged operators' host side without a GPU: exports, every refusal of the C ABI (before
anything is launched), rotary frequencies, and the plan that deals tiles to workgroups."""
import ctypes
import math
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

import paper_2608_14191_amd as P
from paper_2608_14191_amd import _paged
from paper_2608_14191_amd._lib import exported_symbols_declared_in_header

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 5
A, ODD = 1 << 20, (1 << 20) + 1                      # pointers that no refused call follows


def test_exports_and_signatures():
    names = exported_symbols_declared_in_header(os.path.join(ROOT, "include", "aatc_paged.h"))
    assert set(names) == set(_paged._SIGNATURES)
    for n in names:
        assert hasattr(P.library(), n) and hasattr(P, n), n


def _fill(cls, **fields):
    """A structure with plain fields, past its constructor (which takes tensors)."""
    s = cls.__new__(cls)
    ctypes.Structure.__init__(s)
    for k, v in fields.items():
        setattr(s, k, v)
    return s


CACHE = dict(k_pages=A, v_pages=A, dtype=1, n_kv_heads=8, d=128, page_tokens=16, n_pages=100,
             page_stride=8 * 16 * 128, head_stride=16 * 128, tok_stride=128)
TABLE = dict(table=A, stride=32, rows=4, max_pages=32)
ROPE = dict(freq=A, rot_dim=128, layout=0, factor=1.0)

BAD_CACHES = [(dict(k_pages=None), INVALID), (dict(v_pages=None), INVALID), (dict(k_pages=A + 8), INVALID),
              (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(n_kv_heads=0), INVALID),
              (dict(d=64), UNSUPPORTED), (dict(page_tokens=4), INVALID), (dict(page_tokens=24), INVALID),
              (dict(page_tokens=8192), INVALID), (dict(n_pages=0), INVALID), (dict(n_pages=1 << 31), INVALID),
              (dict(page_stride=64), INVALID), (dict(tok_stride=132), INVALID),
              (dict(head_stride=-2048), INVALID), (dict(head_stride=1 << 41), INVALID)]
BAD_TABLES = [(dict(table=None), INVALID), (dict(table=A + 2), INVALID), (dict(rows=0), INVALID),
              (dict(max_pages=0), INVALID), (dict(stride=31), INVALID),
              (dict(rows=1 << 16, max_pages=1 << 15, stride=1 << 15), UNSUPPORTED)]
BAD_ROPES = [(dict(freq=None), INVALID), (dict(freq=A + 4), INVALID), (dict(rot_dim=0), INVALID),
             (dict(rot_dim=63), INVALID), (dict(rot_dim=130), INVALID), (dict(layout=2), INVALID),
             (dict(factor=float("nan")), INVALID), (dict(factor=float("inf")), INVALID)]


def _call(name, args, **change):
    """Calls entry point `name` with the arguments `args` (a dict in order), some changed; struct
    arguments are dicts of (class, fields)."""
    a = dict(args)
    for k, v in change.items():
        assert k in a, k
        a[k] = v
    keep, out = [], []
    for v in a.values():
        if isinstance(v, tuple):
            s = _fill(v[0], **v[1])
            keep.append(s)
            out.append(ctypes.addressof(s))
        else:
            out.append(v)
    return _paged.entry_point(name)(*out)


def _structs(name, args):
    """Every bad structure in the place of each structure argument."""
    kinds = {P.PagedCache: (CACHE, BAD_CACHES), P.PageTable: (TABLE, BAD_TABLES), P.Rope: (ROPE, BAD_ROPES)}
    for k, v in args.items():
        if isinstance(v, tuple):
            good, bads = kinds[v[0]]
            for bad, status in bads:
                assert _call(name, args, **{k: (v[0], {**good, **bad})}) == status, (k, bad)
            if not (name == "aatc_paged_append" and k == "rope"):
                assert _call(name, args, **{k: None}) == INVALID, k


def _each(name, args, refusals):
    for status, change in refusals:
        assert _call(name, args, **change) == status, change


def test_rope_refusals():
    args = dict(x=A, dtype=1, n=0, heads=8, d=128, stride=1024, pos=A, spec=(P.Rope, ROPE), inverse=0,
                out=A, out_stride=1024, stream=None)
    assert _call("aatc_rope", args) == 0                 # no tokens: nothing to do
    _structs("aatc_rope", args)
    _each("aatc_rope", args, [
        (UNSUPPORTED, dict(d=64)), (INVALID, dict(x=None)), (INVALID, dict(out=None)), (INVALID, dict(pos=None)),
        (INVALID, dict(x=ODD)), (INVALID, dict(out=ODD)), (INVALID, dict(pos=A + 2)), (INVALID, dict(dtype=3)),
        (INVALID, dict(dtype=0, x=A + 2)), (INVALID, dict(n=-1)), (INVALID, dict(n=1 << 31)),
        (INVALID, dict(heads=0)), (INVALID, dict(stride=1023)), (INVALID, dict(out_stride=1000)),
        (INVALID, dict(out_stride=2048))])               # in place with another stride


def test_append_refusals():
    args = dict(cache=(P.PagedCache, CACHE), table=(P.PageTable, TABLE), n=0, dtype=1, k=A, ks=1024, v=A,
                vs=1024, seq=A, pos=A, rope=(P.Rope, ROPE), hq=32, q=A, qs=4096, q_out=2 * A, qos=4096,
                stream=None)
    assert _call("aatc_paged_append", args) == 0
    assert _call("aatc_paged_append", args, rope=None, seq=None, hq=0, q=None, q_out=None) == 0
    _structs("aatc_paged_append", args)
    _each("aatc_paged_append", args, [
        (INVALID, dict(n=-1)), (INVALID, dict(n=1 << 31)), (INVALID, dict(dtype=5)), (INVALID, dict(k=None)),
        (INVALID, dict(v=ODD)), (INVALID, dict(ks=1000)), (INVALID, dict(vs=0)), (INVALID, dict(seq=A + 1)),
        (INVALID, dict(pos=None)), (INVALID, dict(hq=0)), (INVALID, dict(q=None)), (INVALID, dict(hq=-1)),
        (INVALID, dict(q_out=None)), (INVALID, dict(qs=4000)), (INVALID, dict(q_out=A, qos=8192))])


ATTEND = dict(cache=(P.PagedCache, CACHE), table=(P.PageTable, TABLE), len=A, batch=4, hq=32, q=A, qd=1,
              qs=4096, scale=0.1, window=0, sink=0, cap=0.0, slopes=None, out=A, lse=None, ws=A,
              ws_bytes=1 << 40, stream=None)


MANY = dict(table=(P.PageTable, {**TABLE, "max_pages": 1 << 24, "stride": 1 << 24}),
            cache=(P.PagedCache, {**CACHE, "page_tokens": 128}))


def test_attention_refusals():
    name = "aatc_paged_decode_attention"
    _structs(name, ATTEND)
    need = P.aatc_paged_decode_workspace_bytes(4, 32, 8)
    nan = float("nan")
    _each(name, ATTEND, [
        (WORKSPACE, dict(ws_bytes=need - 1)), (INVALID, dict(batch=0)), (INVALID, dict(batch=5)),
        (INVALID, dict(hq=0)), (INVALID, dict(hq=30)), (INVALID, dict(len=None)), (INVALID, dict(len=A + 2)),
        (INVALID, dict(q=None)), (INVALID, dict(qd=7)), (INVALID, dict(qs=4095)), (INVALID, dict(q=ODD)),
        (INVALID, dict(scale=nan)), (INVALID, dict(window=-1)), (INVALID, dict(sink=-1)),
        (INVALID, dict(cap=-1.0)), (INVALID, dict(cap=nan)), (INVALID, dict(cap=float("inf"))),
        (INVALID, dict(cap=1e-40)),
        (INVALID, dict(out=None)), (INVALID, dict(out=A + 4)), (INVALID, dict(lse=A + 1)),
        (INVALID, dict(slopes=A + 3)), (INVALID, dict(ws=None)), (INVALID, dict(ws=A + 16))])
    # more tiles than the plan counts: 4 rows of 8 KV heads and 2^24 pages of 128 tokens (2^31
    # tokens, clamped just below) are nearly 2^32 tiles of 16
    assert _call(name, ATTEND, **MANY) == UNSUPPORTED
    for bad in ((0, 32, 8), (4, 0, 8), (4, 32, 0), (4, 30, 8)):
        assert P.aatc_paged_decode_workspace_bytes(*bad) == 0


def test_joined_attention_refusals():
    name = "aatc_decode_attention_paged"
    args = dict(pk=A, pv=A, batch=4, hq=32, hkv=8, d=128, q=A, qd=1, kc=A, ka=A, vc=A, va=A, len=A, cap=1024,
                rk=44, rv=44, scale=0.1, cache=(P.PagedCache, CACHE), table=(P.PageTable, TABLE), plen=A,
                out=A, ws=A, ws_bytes=1 << 40, stream=None)
    _structs(name, args)
    need = P.aatc_decode_paged_workspace_bytes(4, 32, 8, 1024)
    assert need >= P.aatc_decode_workspace_bytes(4, 32, 8, 1024) + P.aatc_paged_decode_workspace_bytes(4, 32, 8)
    _each(name, args, [
        (WORKSPACE, dict(ws_bytes=need - 1)), (WORKSPACE, dict(ws_bytes=16)), (UNSUPPORTED, dict(d=64)),
        (INVALID, dict(batch=5)), (INVALID, dict(batch=0)), (INVALID, dict(hkv=4)), (INVALID, dict(hq=30)),
        (UNSUPPORTED, dict(hq=256)), (INVALID, dict(pk=None)), (INVALID, dict(kc=ODD)), (INVALID, dict(ka=None)),
        (INVALID, dict(len=None)), (INVALID, dict(plen=None)), (INVALID, dict(plen=A + 1)),
        (INVALID, dict(cap=1000)), (INVALID, dict(rk=0)), (INVALID, dict(rv=45)), (INVALID, dict(qd=2)),
        (INVALID, dict(q=ODD)), (INVALID, dict(scale=float("inf"))), (INVALID, dict(out=A + 8)),
        (INVALID, dict(ws=A + 8)), (INVALID, dict(ws=None)), (UNSUPPORTED, MANY)])
    for bad in ((0, 32, 8, 64), (4, 30, 8, 64), (4, 32, 8, -1)):
        assert P.aatc_decode_paged_workspace_bytes(*bad) == 0


def test_page_table_refusals():
    fork = dict(src=(P.PageTable, TABLE), dst=(P.PageTable, TABLE), ref=A, n_pages=100, pairs=A, n=0, stream=None)
    counts = [(INVALID, dict(ref=None)), (INVALID, dict(ref=A + 2)), (INVALID, dict(n_pages=0)),
              (INVALID, dict(n_pages=1 << 31))]
    assert _call("aatc_pages_fork", fork) == 0
    _structs("aatc_pages_fork", fork)
    _each("aatc_pages_fork", fork, counts + [
        (INVALID, dict(pairs=None)), (INVALID, dict(pairs=A + 2)), (INVALID, dict(n=-1)), (INVALID, dict(n=1 << 31)),
        (UNSUPPORTED, dict(n=1 << 24)), (INVALID, dict(dst=(P.PageTable, {**TABLE, "max_pages": 31})))])
    free = dict(table=(P.PageTable, TABLE), ref=A, n_pages=100, rows=A, n=0, stream=None)
    assert _call("aatc_pages_free", free) == 0
    _structs("aatc_pages_free", free)
    _each("aatc_pages_free", free, counts + [(INVALID, dict(rows=None)), (INVALID, dict(n=-1)), (UNSUPPORTED, dict(n=1 << 24))])
    need = P.aatc_pages_workspace_bytes(4, 100)
    reserve = dict(table=(P.PageTable, TABLE), ref=A, n_pages=100, page=16, held=A, wanted=A, pairs=A,
                   lacking=A, ws=A, ws_bytes=1 << 40, stream=None)
    _structs("aatc_pages_reserve", reserve)
    _each("aatc_pages_reserve", reserve, counts + [
        (INVALID, dict(page=12)), (INVALID, dict(page=4)), (INVALID, dict(page=1 << 13)), (INVALID, dict(held=None)),
        (INVALID, dict(wanted=A + 1)), (INVALID, dict(pairs=None)), (INVALID, dict(lacking=None)),
        (INVALID, dict(ws=None)), (INVALID, dict(ws=A + 8)), (WORKSPACE, dict(ws_bytes=need - 1))])
    compact = dict(table=(P.PageTable, TABLE), ref=A, n_pages=100, out=(P.PageTable, TABLE), ref_out=A, pairs=A,
                   moves=A, ws=A, ws_bytes=1 << 40, stream=None)
    _structs("aatc_pages_compact", compact)
    _each("aatc_pages_compact", compact, counts + [
        (INVALID, dict(ref_out=None)), (INVALID, dict(pairs=None)), (INVALID, dict(moves=A + 2)),
        (INVALID, dict(out=(P.PageTable, {**TABLE, "rows": 3}))), (INVALID, dict(ws=A + 4)),
        (INVALID, dict(out=(P.PageTable, {**TABLE, "stride": 40}))), (WORKSPACE, dict(ws_bytes=need - 1))])
    copy = dict(base=A, pools=2, stride=16000, n_pages=100, page=160, pairs=A, n=0, n_dev=None, stream=None)
    assert _call("aatc_pages_copy", copy) == 0
    _each("aatc_pages_copy", copy, [
        (INVALID, dict(base=None)), (INVALID, dict(base=A + 8)), (INVALID, dict(pools=0)), (INVALID, dict(n_pages=0)),
        (INVALID, dict(page=8)), (INVALID, dict(page=24)), (INVALID, dict(stride=15984)), (INVALID, dict(n=-1)),
        (INVALID, dict(n=5, pairs=None)), (INVALID, dict(pairs=A + 2)), (INVALID, dict(n_dev=A + 1)),
        (INVALID, dict(stride=16008))])
    for bad in ((0, 5), (5, 0), (-1, 5)):
        assert P.aatc_pages_workspace_bytes(*bad) == 0


# -------------------------------------------------------------------- rotary frequencies
def test_frequencies():
    for rot in (2, 50, 128):
        f, factor = P.aatc_rope_frequencies(rot, 10000.0)
        want = 10000.0 ** (-np.arange(0, rot, 2) / rot)
        np.testing.assert_allclose(f, want, rtol=1e-14)
        assert factor == 1.0
    rot, base, scale, trained = 128, 500000.0, 8.0, 8192
    plain = base ** (-np.arange(0, rot, 2) / rot)
    f, factor = P.aatc_rope_frequencies(rot, base, P.ROPE_LINEAR, scale)
    np.testing.assert_allclose(f, plain / scale, rtol=1e-14)
    f, _ = P.aatc_rope_frequencies(rot, base, P.ROPE_NTK, scale)
    np.testing.assert_allclose(f, (base * scale ** (rot / (rot - 2))) ** (-np.arange(0, rot, 2) / rot), rtol=1e-13)
    np.testing.assert_allclose(f[-1], plain[-1] / scale, rtol=1e-13)     # the slowest pair: as LINEAR
    f, factor = P.aatc_rope_frequencies(rot, base, P.ROPE_BANDS, scale, trained, 1.0, 4.0)
    turns = trained * plain / (2 * math.pi)
    keep = np.clip((turns - 1) / 3, 0, 1)
    np.testing.assert_allclose(f, plain * keep + plain / scale * (1 - keep), rtol=1e-13)
    # (two libraries' powers, each within an ulp, and a division: 3 2^-53 relative)
    np.testing.assert_allclose(f[turns <= 1], plain[turns <= 1] / scale, rtol=1e-15)
    assert f[0] == plain[0] and factor == 1.0
    f, factor = P.aatc_rope_frequencies(rot, base, P.ROPE_YARN, scale, trained, 1.0, 32.0)
    at = lambda u: rot * math.log(trained / (u * 2 * math.pi)) / (2 * math.log(base))       # noqa: E731
    lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
    keep = 1 - np.clip((np.arange(rot // 2) - lo) / (hi - lo), 0, 1)
    np.testing.assert_allclose(f, plain * keep + plain / scale * (1 - keep), rtol=1e-13)
    assert abs(factor - (0.1 * math.log(8) + 1)) < 1e-6
    # scale 1 changes nothing
    for kind in (P.ROPE_LINEAR, P.ROPE_NTK, P.ROPE_BANDS, P.ROPE_YARN):
        f, factor = P.aatc_rope_frequencies(rot, base, kind, 1.0, trained, 1.0, 4.0)
        np.testing.assert_allclose(f, plain, rtol=1e-13)
        assert factor == 1.0


@pytest.mark.parametrize("args", [(0, 1e4), (3, 1e4), (130, 1e4), (64, 1.0), (64, float("nan")), (64, float("inf")),
                                  (64, 1e4, 5), (64, 1e4, -1), (64, 1e4, P.ROPE_LINEAR, 0.5),
                                  (64, 1e4, P.ROPE_LINEAR, float("nan")), (2, 1e4, P.ROPE_NTK, 2.0),
                                  (64, 1e4, P.ROPE_BANDS, 2.0, 0), (64, 1e4, P.ROPE_BANDS, 2.0, 100, 0.0, 4.0),
                                  (64, 1e4, P.ROPE_YARN, 2.0, 100, 4.0, 4.0)])
def test_frequency_refusals(args):
    with pytest.raises(P.AatcError) as e:
        P.aatc_rope_frequencies(*args)
    assert e.value.status == INVALID


# ------------------------------------------------------------------------------- plan
@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host C++ compiler")
    lib = tmp_path_factory.mktemp("plan") / "plan.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2608_14191_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "paged_plan_harness.cpp"), "-o", str(lib)], check=True)
    return ctypes.CDLL(str(lib))


def _tiles(plan, n, window, sink, tt):
    room = max(1, -(-n // tt))
    out = (ctypes.c_int * room)()
    got = plan.tiles(n, window, sink, tt, out, room)
    assert 1 <= got <= room
    return list(out)[:got]


def test_tiles_hold_every_attended_token_once(plan):
    r = random.Random(3)
    for _ in range(3000):
        tt = r.choice([16, 32])
        n = r.choice([0, 1, 31, 32, 33, r.randint(0, 400), r.randint(0, 3000)])
        window = r.choice([0, 0, 1, r.randint(1, 64), r.randint(1, 3000)])
        sink = r.choice([0, 4, r.randint(0, 64), r.randint(0, 3000)])
        starts = _tiles(plan, n, window, sink, tt)
        assert starts == sorted(set(starts)) and all(t % tt == 0 for t in starts)
        want = {t // tt for t in range(n) if window == 0 or t >= n - window or t < sink}
        assert {t // tt for t in starts} == (want or {0})


def test_runs_fit_the_grid(plan):
    r = random.Random(4)
    for _ in range(2000):
        rows = r.choice([1, 1, 4, 8, 16])
        batch = r.randint(1, r.choice([128, 256]) // rows)
        most = r.choice([1, 5, 60, 700, 4096])
        n = [r.randint(1, most) for _ in range(batch)]
        q = 8 * plan.rounds((ctypes.c_int * batch)(*n), batch, rows, 256, 8)
        runs = [-(-x // q) for x in n]
        assert rows * sum(runs) <= 256
        for x, k in zip(n, runs):
            cuts = [plan.run_at(x, k, i) for i in range(k + 1)]
            assert cuts[0] == 0 and cuts[-1] == x
            assert all(0 < b - a <= q for a, b in zip(cuts, cuts[1:]))
        # not much longer than they need to be: an eighth and two rounds shorter would not fit
        if q > 32:
            assert rows * sum(-(-x // (q - q // 8 - 16)) for x in n) > 256


def test_lines_cover_every_tile_once_with_parts_of_their_own(plan):
    r = random.Random(5)
    for _ in range(300):
        rows = r.randint(129, 700)
        most = r.choice([1, 3, 12, 60, 500])
        n = [r.randint(1, most) for _ in range(rows)]
        total, out = sum(n), (ctypes.c_int * 3)()
        plan.way(total, max(n), rows, 512, 4, out)
        quota, waves, whole = out
        workers = 512 * 4 if waves else 512
        if whole:
            assert rows <= workers and quota >= max(n)
            continue
        assert quota * workers >= total
        start, used, taken = 0, set(), {}
        for x in n:
            out2 = (ctypes.c_int * 2)()
            plan.share(start, x, quota, out2)
            first, last = out2
            assert 0 <= first <= last < workers
            if waves:
                assert last - first + 1 <= 16          # parts that one wave joins
            for w in range(first, last + 1):
                a, b = max(start, w * quota), min(start + x, (w + 1) * quota)
                assert b > a
                taken[w] = taken.get(w, 0) + b - a
                if last > first:
                    slot = plan.slot(w, start, quota)
                    assert 0 <= slot < 2 * workers and slot not in used
                    used.add(slot)
            start += x
        assert sum(taken.values()) == total and max(taken.values()) <= quota
