"""The operators over 8-bit pages, under a window and of forks refuse bad arguments before they touch the device (fake
pointers that nothing follows)."""
import ctypes

import pytest

from paper_2609_17184_amd import binding as B
from test_serving_cpu import BAD_BATCH, BAD_CACHE, FAKE, _attn, _batch, _cache, _rope


def _scales(**kw):
    s = dict(k=FAKE, v=FAKE, k_page=2, k_head=1, v_page=2, v_head=1)
    s.update(kw)
    return B.PageScalesC(**s)


def _append_rc(c, s, b, a):
    return B.load_library().loopspec_rope_append_quantized(ctypes.byref(c), ctypes.byref(s), ctypes.byref(b), ctypes.byref(a), None)


def _window_rc(c, s, b, a, window=10, sinks=2, ws=FAKE, nbytes=1 << 40):
    return B.load_library().loopspec_window_attention(ctypes.byref(c), None if s is None else ctypes.byref(s), ctypes.byref(b),
                                                      ctypes.byref(a), window, sinks, ws, nbytes, None)


def _need(c, s, b, heads=4, window=10, sinks=2):
    return B.load_library().loopspec_window_attention_workspace_bytes(
        ctypes.byref(c), None if s is None else ctypes.byref(s), ctypes.byref(b), heads, window, sinks)


@pytest.mark.parametrize("bad", BAD_CACHE + [dict(k_page=2056), dict(v_pos=72), dict(k_head=1032)], ids=str)
def test_bad_caches(bad):
    assert _append_rc(_cache(**bad), _scales(), _batch(), _rope()) == B.EINVAL
    assert _window_rc(_cache(**bad), _scales(), _batch(), _attn()) == B.EINVAL
    assert _need(_cache(**bad), _scales(), _batch(table_width=1000, table_stride=1000), window=0) == 0


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(k_page=-1), dict(v_page=0), dict(k_head=0), dict(v_head=-1)], ids=str)
def test_bad_scales(bad):
    assert _append_rc(_cache(), _scales(**bad), _batch(), _rope()) == B.EINVAL
    assert _window_rc(_cache(), _scales(**bad), _batch(), _attn()) == B.EINVAL
    assert B.load_library().loopspec_rope_append_quantized(ctypes.byref(_cache()), None, ctypes.byref(_batch()), ctypes.byref(_rope()), None) == B.EINVAL


@pytest.mark.parametrize("bad", BAD_BATCH, ids=str)
def test_bad_batches(bad):
    assert _append_rc(_cache(), _scales(), _batch(**bad), _rope()) == B.EINVAL
    for s in (None, _scales()):
        assert _window_rc(_cache(), s, _batch(**bad), _attn()) == B.EINVAL


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_heads=3), dict(rot_dim=24), dict(rot_dim=80), dict(freq=None),
                                 dict(eps=float("nan")), dict(q=None), dict(k=FAKE + 4), dict(v_head=4), dict(out_head=32)], ids=str)
def test_bad_append(bad):
    assert _append_rc(_cache(), _scales(), _batch(), _rope(**bad)) == B.EINVAL


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_heads=5), dict(scale=0.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(q=None), dict(out=None), dict(q=FAKE + 2), dict(q_head=12),
                                 dict(out_token=8)], ids=str)
def test_bad_attention(bad):
    for s in (None, _scales()):
        assert _window_rc(_cache(), s, _batch(), _attn(**bad)) == B.EINVAL


def test_windows_workspaces_and_grids():
    for kw in (dict(window=-1), dict(sinks=-1)):
        assert _window_rc(_cache(), None, _batch(), _attn(), **kw) == B.EINVAL and _need(_cache(), None, _batch(), **kw) == 0
    wide = _batch(table_width=4000, table_stride=4000)
    need = _need(_cache(), None, wide, window=0)
    assert need > 0 and _need(_cache(), None, wide) == 0               # under a short window one workgroup has all of a row
    for kw in (dict(nbytes=need - 1), dict(ws=None), dict(ws=FAKE + 4)):
        assert _window_rc(_cache(), None, wide, _attn(), window=0, **kw) == B.EINVAL
    assert _window_rc(_cache(), None, _batch(prefix_table=None), _attn()) == B.EINVAL
    big = _batch(n_tokens=(1 << 23) + 1, n_seqs=1 << 23)
    assert _window_rc(_cache(), None, big, _attn(), nbytes=1 << 62) == B.EINVAL


def test_nothing_to_do():
    none = dict(q=None, k=None, v=None, q_out=None)
    for kw in (dict(n_seqs=0), dict(n_tokens=0)):
        assert _append_rc(_cache(), _scales(), _batch(**kw), _rope(**none)) == B.OK
        assert _window_rc(_cache(), _scales(), _batch(**kw), _attn(q=None, out=None), ws=None, nbytes=0) == B.OK


def _fork(**kw):
    a = dict(n_seqs=2, n_children=3, page_size=16, n_pages=10, seq_len=FAKE, table=FAKE, table_stride=4, table_width=4,
             parent=FAKE, refs=FAKE, prefix_len=0, window=0, sinks=0, room=0, seq_len_out=FAKE, table_out=FAKE, out_stride=4,
             refs_out=FAKE, short=FAKE)
    a.update(kw)
    return B.ForkArgs(**a)


def _fork_rc(a, caches=None, scales=None, n=1, ws=FAKE, nbytes=1 << 30):
    caches = (B.PagedCacheC * 1)(_cache()) if caches is None else caches
    return B.load_library().loopspec_fork_pages(ctypes.byref(a), caches, scales, n, ws, nbytes, None)


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=65536), dict(n_children=-1), dict(n_children=65536), dict(page_size=24),
                                 dict(page_size=0), dict(n_pages=0), dict(n_pages=11), dict(seq_len=None), dict(table=None),
                                 dict(table_stride=3), dict(table_width=-1), dict(table_width=1 << 25, table_stride=1 << 25, out_stride=1 << 25),
                                 dict(n_children=65535, table_width=1 << 16, table_stride=1 << 16, out_stride=1 << 16),
                                 dict(parent=None), dict(refs=None), dict(prefix_len=-1), dict(window=-1), dict(sinks=-1), dict(room=-1),
                                 dict(room=65), dict(seq_len_out=None), dict(table_out=None), dict(out_stride=3), dict(refs_out=None),
                                 dict(short=None)], ids=str)
def test_bad_forks(bad):
    assert _fork_rc(_fork(**bad)) == B.EINVAL


def test_bad_fork_caches_and_workspaces():
    need = B.load_library().loopspec_fork_pages_workspace_bytes(3, 10)
    assert need > 0 and B.load_library().loopspec_fork_pages_workspace_bytes(-1, 10) == 0
    assert B.load_library().loopspec_fork_pages_workspace_bytes(3, 0) == 0
    for kw in (dict(nbytes=need - 1), dict(ws=None), dict(ws=FAKE + 4), dict(n=-1)):
        assert _fork_rc(_fork(), **kw) == B.EINVAL
    for bad in (dict(page_size=32), dict(n_pages=9), dict(k=None), dict(k_pos=8)):
        assert _fork_rc(_fork(), (B.PagedCacheC * 1)(_cache(**bad))) == B.EINVAL
    for bad in (dict(v=None), dict(k_head=-1)):
        assert _fork_rc(_fork(), scales=(B.PageScalesC * 1)(_scales(**bad))) == B.EINVAL
    assert _fork_rc(_fork(), (B.PagedCacheC * 1)(_cache(v_head=1032)), scales=(B.PageScalesC * 1)(_scales())) == B.EINVAL
    assert B.load_library().loopspec_fork_pages(None, None, None, 0, FAKE, 1 << 30, None) == B.EINVAL
    assert B.load_library().loopspec_fork_pages(ctypes.byref(_fork()), None, None, 1, FAKE, 1 << 30, None) == B.EINVAL
