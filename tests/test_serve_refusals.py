"""What the entry points around the reduction refuse, on the host and before anything is launched.  CPU only: the pointers below
are never read."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def dart():
    from paper_2502_11494_b200 import build, dart as d

    build.build_library()
    return d


A, B, C, D_ = 1 << 20, 1 << 24, 1 << 28, 1 << 29  # addresses far apart


def _rope(dart, **kw):
    r = dict(inv_freq=A, rot_dim=64, interleaved=0, n_axes=1, section=(0, 0, 0))
    r.update(kw)
    return dart.dart_rope(r["inv_freq"], r["rot_dim"], r["interleaved"], r["n_axes"], (ctypes.c_int32 * 3)(*r["section"]))


def _norm_rope(dart, **kw):
    a = dict(q=A, qs=512, hq=4, k=B, ks=256, hk=2, n=8, D=128, dtype=0, wq=None, wk=None, eps=1e-6, rope=None, pos=A, ps=64, qo=C, qos=512,
             ko=D_, kos=256)
    a.update(kw)
    return dart.dart_norm_rope(a["q"], a["qs"], a["hq"], a["k"], a["ks"], a["hk"], a["n"], a["D"], a["dtype"], a["wq"], a["wk"], a["eps"],
                               a["rope"], a["pos"], a["ps"], a["qo"], a["qos"], a["ko"], a["kos"], 0, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), 0), (dict(n=0, q=None), 0),
    (dict(n=-1), -2), (dict(hq=0, hk=0), -2), (dict(hq=-1), -2), (dict(D=0), -2), (dict(D=12), -2), (dict(D=264), -2),
    (dict(eps=-1.0), -2), (dict(eps=float("nan")), -2), (dict(eps=float("inf")), -2), (dict(qs=504), -2), (dict(qs=516), -2), (dict(kos=128), -2),
    (dict(hq=65536), -2), (dict(dtype=2), -9), (dict(dtype=-1), -9),
    (dict(q=None), -1), (dict(ko=None), -1),
    (dict(q=A + 8), -3), (dict(ko=D_ + 2), -3), (dict(wq=A + 4), -3),
    (dict(qo=A + 16), -4), (dict(qo=A, qos=1024), -4), (dict(qo=B), -4), (dict(ko=C), -4), (dict(ko=A), -4), (dict(qo=B + 1024), -4),
])
def test_norm_rope_refuses(dart, kw, code):
    assert _norm_rope(dart, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(inv_freq=None), -1), (dict(rot_dim=8), -2), (dict(rot_dim=144), -2), (dict(rot_dim=-16), -2),
    (dict(n_axes=4), -2), (dict(n_axes=-1), -2), (dict(n_axes=3, section=(8, 8, 8)), -2), (dict(n_axes=3, section=(40, 8, -16)), -2),
    (dict(inv_freq=A + 2), -3),
])
def test_rotations_that_are_refused(dart, kw, code):
    assert _norm_rope(dart, rope=_rope(dart, **kw)) == code


def test_positions_that_are_refused(dart):
    assert _norm_rope(dart, rope=_rope(dart), pos=None) == dart.DART_ERR_NULL
    assert _norm_rope(dart, rope=_rope(dart), pos=A + 4) == dart.DART_ERR_ALIGN
    assert _norm_rope(dart, rope=_rope(dart, n_axes=2, section=(16, 16, 0)), ps=7) == dart.DART_ERR_BAD_SHAPE
    assert _norm_rope(dart, rope=_rope(dart, rot_dim=0), pos=None, n=0) == dart.DART_OK


def test_columns_of_one_buffer_are_no_overlap(dart):
    """Queries and keys side by side in a projection's output, and the results side by side in another: only the device is missing."""
    got = _norm_rope(dart, q=A, qs=1024, k=A + 2 * 512, ks=1024, qo=C, qos=1024, ko=C + 2 * 512, kos=1024)
    assert got in (dart.DART_OK, dart.DART_ERR_CUDA) and got != dart.DART_ERR_ALIAS
    in_place = _norm_rope(dart, q=A, qs=1024, k=A + 2 * 512, ks=1024, qo=A, qos=1024, ko=A + 2 * 512, kos=1024, n=8)
    assert in_place != dart.DART_ERR_ALIAS
    assert _norm_rope(dart, q=A, qs=1024, k=A + 2 * 504, ks=1024, qo=A, qos=1024, ko=C, kos=256) == dart.DART_ERR_ALIAS


def _append(dart, cache=None, **kw):
    c = dict(k=C, v=D_, n_pages=16, n_heads=2, page_size=16, head_dim=128, dtype=0, device=0)
    c.update(cache or {})
    a = dict(k=A, ks=256, v=B, vs=256, n_seq=2, n=8, cu=None, idx=None, S=0, table=A, ts=4, start=None, wk=None, eps=1e-6, rope=None, pos=None, ps=0, status=None)
    a.update(kw)
    return dart.dart_cache_append(dart.dart_cache(*c.values()), a["k"], a["ks"], a["v"], a["vs"], a["n_seq"], a["n"], a["cu"], a["idx"], a["S"],
                                  a["table"], a["ts"], a["start"], a["wk"], a["eps"], a["rope"], a["pos"], a["ps"], a["status"], None)


@pytest.mark.parametrize("cache,kw,code", [
    ({}, dict(n=0), 0), ({}, dict(n=0, k=None), 0),
    (dict(k=None), {}, -1), (dict(n_pages=0), {}, -2), (dict(n_heads=0), {}, -2), (dict(page_size=0), {}, -2), (dict(head_dim=100), {}, -2),
    (dict(head_dim=264), {}, -2), (dict(dtype=5), {}, -9), (dict(k=C + 8), {}, -3),
    ({}, dict(n=7), -2), ({}, dict(n=-2), -2), ({}, dict(n_seq=0), -2), ({}, dict(ts=0), -2), ({}, dict(idx=A, S=0), -2), ({}, dict(ks=248), -2),
    ({}, dict(k=None), -1), ({}, dict(table=None), -1), ({}, dict(v=B + 4), -3), ({}, dict(table=A + 2), -3), ({}, dict(status=A + 1), -3),
    ({}, dict(k=C + 4096), -4), ({}, dict(v=D_), -4), (dict(v=C + 1024), {}, -4),
])
def test_append_refuses(dart, cache, kw, code):
    assert _append(dart, cache, **kw) == code


def test_append_takes_slots_as_positions_on_one_axis_only(dart):
    assert _append(dart, rope=_rope(dart, n_axes=3, section=(16, 8, 8))) == dart.DART_ERR_NULL
    assert dart.dart_cache_append(None, A, 256, B, 256, 1, 1, None, None, 0, A, 1, None, None, 0.0, None, None, 0, None, None) == dart.DART_ERR_NULL


def test_struct_layouts(dart):
    assert ctypes.sizeof(dart.dart_rope) == 32 and dart.dart_rope.rot_dim.offset == 8 and dart.dart_rope.section.offset == 20
    assert ctypes.sizeof(dart.dart_cache) == 40 and dart.dart_cache.n_pages.offset == 16


def _attend(dart, cache=None, ws=1 << 30, ws_bytes=1 << 40, **kw):
    c = dict(k=C, v=D_, n_pages=16, n_heads=2, page_size=16, head_dim=128, dtype=0, device=0)
    c.update(cache or {})
    a = dict(q=A, out=B, lse=None, q_stride=1024, out_stride=1024, n_rows=4, n_q_heads=8, n_seq=4, n_groups=0, cu_q=None, table=A, kv_len=A, cu_group=None,
             prefix_table=None, prefix_len=None, table_stride=4, prefix_stride=0, scale=0.1, wait_limit=0, status=None, test_withhold=0)
    a.update(kw)
    cache, args = dart.dart_cache(*c.values()), dart.dart_attend_args(*a.values())
    return dart.dart_attend(cache, args, ws, ws_bytes, None), dart.dart_attend_workspace(cache, args)


GROUPS = dict(n_groups=2, cu_group=A, prefix_table=A, prefix_len=A, prefix_stride=4)


@pytest.mark.parametrize("cache,kw,code", [
    (dict(v=None), {}, -1), (dict(head_dim=96), {}, -9), (dict(head_dim=256), {}, -9), (dict(page_size=8), {}, -9), (dict(page_size=48), {}, -9),
    (dict(page_size=2048), {}, -9), (dict(dtype=3), {}, -9), (dict(n_pages=0), {}, -2), (dict(n_pages=1 << 27), {}, -2), (dict(v=D_ + 8), {}, -3),
    ({}, dict(n_rows=-1), -2), ({}, dict(n_seq=0), -2), ({}, dict(n_groups=-1), -2), ({}, dict(n_q_heads=0), -2), ({}, dict(n_q_heads=7), -2), ({}, dict(table_stride=0), -2),
    ({}, dict(scale=0.0), -2), ({}, dict(scale=-1.0), -2), ({}, dict(scale=float("nan")), -2), ({}, dict(scale=float("inf")), -2), ({}, dict(n_rows=5), -2),
    ({}, dict(wait_limit=-1), -2), ({}, dict(q_stride=1016), -2), ({}, dict(out_stride=1020), -2), ({}, dict(n_rows=1 << 28, cu_q=A), -2), ({}, dict(table_stride=1 << 28), -2),
    ({}, dict(GROUPS, prefix_stride=0), -2), ({}, dict(GROUPS, prefix_len=None), -1), ({}, dict(GROUPS, cu_group=None), -1),
    ({}, dict(q=None), -1), ({}, dict(out=None), -1), ({}, dict(table=None), -1), ({}, dict(kv_len=None), -1), ({}, dict(q=A + 8), -3), ({}, dict(out=B + 8), -3),
    ({}, dict(kv_len=A + 2), -3), ({}, dict(status=A + 3), -3), ({}, dict(lse=A + 2), -3),
    ({}, dict(out=A), -4), ({}, dict(out=C), -4), ({}, dict(out=D_ + 16), -4), ({}, dict(lse=B), -4), ({}, dict(lse=A + 1024), -4), ({}, dict(lse=C), -4),
])
def test_attend_refuses(dart, cache, kw, code):
    assert _attend(dart, cache, **kw) == (code, 0)


def test_attend_wants_its_workspace(dart):
    rc, need = _attend(dart, ws_bytes=255)
    assert rc == dart.DART_ERR_NOMEM and need > 255 and need % 256 == 0
    assert _attend(dart, ws=None)[0] == dart.DART_ERR_NULL and _attend(dart, ws=(1 << 30) + 128)[0] == dart.DART_ERR_ALIGN
    assert _attend(dart, n_rows=0, cu_q=A) == (dart.DART_OK, 0) and _attend(dart, **GROUPS)[1] > need
    assert dart.dart_attend(None, None, None, 0, None) == dart.DART_ERR_NULL
    assert ctypes.sizeof(dart.dart_attend_args) == 136 and dart.dart_attend_args.scale.offset == 112 and dart.dart_attend_args.status.offset == 120


def test_rows_of_a_table_end_inside_its_memory(dart):
    """The kernels take a row of a table for as wide as its stride, and cut lengths at that: columns of a wider table from the first one on are
    taken as they lie, later ones, whose last row would end beyond the memory, are copied."""
    torch = pytest.importorskip("torch")
    cache = object.__new__(dart.PagedCache)
    cache._int32, cache.device = torch.int32, torch.device("cpu")
    wide = torch.arange(40, dtype=torch.int32).view(4, 10)
    views = [wide, wide[:, :6], wide[:, 5:], wide[1:, 3:], wide[:3, 5:], wide[3:, 2:5], wide[:, 9:], wide.view(-1)[2:38].view(4, 9), wide[::2], wide[::3, 4:]]
    copied = []
    for v in views:
        at, stride, rows, keep = cache._table(v, "table")
        end = keep.untyped_storage().data_ptr() + keep.untyped_storage().nbytes()
        assert rows == v.shape[0] and at == keep.data_ptr() and at + 4 * stride * rows <= end and stride >= v.shape[1] and torch.equal(keep, v)
        copied.append(at != v.data_ptr())
    assert copied == [False, False, True, True, False, False, True, False, False, True]
