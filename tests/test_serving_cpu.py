"""The serving operators refuse bad arguments before they touch the device (fake pointers that nothing follows)."""
import ctypes

import pytest

from paper_2609_17184_amd import binding as B
from paper_2609_17184_amd import serving

FAKE = 1 << 20


def _cache(**kw):
    c = dict(dtype=B.F16, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, k=FAKE, v=FAKE, k_page=2048, k_head=1024,
             k_pos=64, v_page=2048, v_head=1024, v_pos=64)
    c.update(kw)
    return B.PagedCacheC(**c)


def _batch(**kw):
    b = dict(n_seqs=2, n_tokens=2, q_start=None, seq_len=FAKE, table=FAKE, table_stride=4, table_width=4, prefix_len=20,
             prefix_table=FAKE)
    b.update(kw)
    return B.PagedBatchC(**b)


def _rope(**kw):
    a = dict(n_heads=4, rot_dim=64, eps=1e-6, q=FAKE, k=FAKE, v=FAKE, q_token=256, q_head=64, k_token=128, k_head=64,
             v_token=128, v_head=64, q_out=FAKE, out_token=256, out_head=64, freq=FAKE, q_norm=None, k_norm=None)
    a.update(kw)
    return B.RopeArgs(**a)


def _attn(**kw):
    a = dict(n_heads=4, scale=0.125, q=FAKE, q_token=256, q_head=64, out=FAKE, out_token=256, out_head=64, lse=None)
    a.update(kw)
    return B.AttentionArgs(**a)


BAD_CACHE = [dict(dtype=B.F32), dict(dtype=9), dict(n_pages=0), dict(page_size=8), dict(page_size=24),
             dict(page_size=2048), dict(page_size=0), dict(n_kv_heads=0), dict(head_dim=48), dict(head_dim=256),
             dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(v=FAKE + 8), dict(k_page=2050), dict(v_head=1028),
             dict(k_pos=32), dict(v_pos=-64), dict(k_head=0), dict(v_page=8), dict(k_pos=1 << 25)]
BAD_BATCH = [dict(n_seqs=-1), dict(n_tokens=-1), dict(seq_len=None), dict(table=None), dict(table_stride=3),
             dict(table_width=-1), dict(prefix_len=-1), dict(prefix_len=(1 << 28) + 1), dict(table_width=1 << 25),
             dict(n_tokens=(1 << 25) + 1)]


def _rope_rc(c, b, a):
    return B.load_library().loopspec_rope_append(ctypes.byref(c), ctypes.byref(b), ctypes.byref(a), None)


def _attn_rc(c, b, a, ws=FAKE, nbytes=1 << 40):
    return B.load_library().loopspec_prefix_attention(ctypes.byref(c), ctypes.byref(b), ctypes.byref(a), ws, nbytes, None)


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_bad_caches(bad):
    assert _rope_rc(_cache(**bad), _batch(), _rope()) == B.EINVAL
    assert _attn_rc(_cache(**bad), _batch(), _attn()) == B.EINVAL
    assert B.load_library().loopspec_prefix_attention_workspace_bytes(
        ctypes.byref(_cache(**bad)), ctypes.byref(_batch()), 4) == 0


@pytest.mark.parametrize("bad", BAD_BATCH, ids=str)
def test_bad_batches(bad):
    assert _rope_rc(_cache(), _batch(**bad), _rope()) == B.EINVAL
    assert _attn_rc(_cache(), _batch(**bad), _attn()) == B.EINVAL


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_heads=3), dict(rot_dim=-16), dict(rot_dim=24),
                                 dict(rot_dim=80), dict(freq=None), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(q=FAKE + 4),
                                 dict(k_token=100), dict(v_head=4), dict(q_token=-256), dict(out_head=32),
                                 dict(out_token=0)], ids=str)
def test_bad_append(bad):
    assert _rope_rc(_cache(), _batch(), _rope(**bad)) == B.EINVAL


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_heads=5), dict(scale=0.0), dict(scale=-1.0),
                                 dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None),
                                 dict(out=None), dict(q=FAKE + 2), dict(q_head=12), dict(out_token=8), dict(out_head=0)],
                         ids=str)
def test_bad_attention(bad):
    assert _attn_rc(_cache(), _batch(), _attn(**bad)) == B.EINVAL


def test_attention_grids():
    """More rows than the grids hold."""
    big = _batch(n_tokens=(1 << 23) + 1, n_seqs=1 << 23)
    assert _attn_rc(_cache(), big, _attn(), nbytes=1 << 62) == B.EINVAL
    assert B.load_library().loopspec_prefix_attention_workspace_bytes(ctypes.byref(_cache()), ctypes.byref(big), 4) == 0


def test_attention_workspace():
    L = B.load_library()
    need = L.loopspec_prefix_attention_workspace_bytes(ctypes.byref(_cache()), ctypes.byref(_batch()), 4)
    assert need > 0
    assert _attn_rc(_cache(), _batch(), _attn(), nbytes=need - 1) == B.EINVAL
    assert _attn_rc(_cache(), _batch(), _attn(), ws=None) == B.EINVAL
    assert _attn_rc(_cache(), _batch(), _attn(), ws=FAKE + 4) == B.EINVAL
    assert _attn_rc(_cache(), _batch(prefix_table=None), _attn()) == B.EINVAL


def test_nothing_to_do():
    """No sequences or no tokens: no launch (none would succeed here), and addresses do not matter, as empty tensors
    have none."""
    none = dict(q=None, k=None, v=None, q_out=None)
    assert _rope_rc(_cache(), _batch(n_tokens=0), _rope(**none)) == B.OK
    assert _attn_rc(_cache(), _batch(n_tokens=0), _attn(q=None, out=None), ws=None, nbytes=0) == B.OK
    cfg = B.SampleCfg(100, B.F32, 1.0, 0, 1.0, 0.0)
    assert B.load_library().loopspec_sample(ctypes.byref(cfg), 0, None, 100, None, None, None, None, None, 0, None) == B.OK
    for kw in (dict(n_seqs=0), dict(n_tokens=0)):
        assert _rope_rc(_cache(), _batch(**kw), _rope()) == B.OK
        assert _attn_rc(_cache(), _batch(**kw), _attn(), ws=None, nbytes=0) == B.OK
    for i in range(3):
        args = [ctypes.byref(x) for x in (_cache(), _batch(), _rope())]
        args[i] = None
        assert B.load_library().loopspec_rope_append(*args, None) == B.EINVAL


def test_binding_checks_tensors():
    import torch
    k = torch.zeros((4, 2, 16, 64), dtype=torch.float16)
    for kk, vv in ((k, k), (k[0], k[0]), (k, k.float()), (k.float(), k.float())):
        with pytest.raises(ValueError):
            serving.PagedCache(kk, vv)                      # host memory, shape, types
    with pytest.raises(ValueError):
        serving.Batch(torch.zeros(3, dtype=torch.int32), torch.zeros((3, 4), dtype=torch.int32))


def _sample_rc(rows=4, logits=FAKE, stride=1000, u=FAKE, token=FAKE, ws=FAKE, nbytes=1 << 40, **kw):
    c = dict(vocab=1000, dtype=B.F32, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    c.update(kw)
    cfg = B.SampleCfg(**c)
    return B.load_library().loopspec_sample(ctypes.byref(cfg), rows, logits, stride, u, token, None, None, ws,
                                            nbytes, None)


@pytest.mark.parametrize("bad", [dict(vocab=0), dict(vocab=262145), dict(dtype=3), dict(temperature=-0.5),
                                 dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_p=0.0),
                                 dict(top_p=1.5), dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.1),
                                 dict(rows=-1), dict(rows=65536), dict(ws=None), dict(ws=FAKE + 8), dict(nbytes=1000), dict(logits=None), dict(logits=FAKE + 2), dict(stride=-1), dict(u=None),
                                 dict(token=None)], ids=str)
def test_bad_samples(bad):
    assert _sample_rc(**bad) == B.EINVAL


def test_sample_of_no_rows():
    assert _sample_rc(rows=0) == B.OK
    assert B.load_library().loopspec_sample(None, 1, FAKE, 10, FAKE, FAKE, None, None, FAKE, 1 << 40, None) == B.EINVAL
    L = B.load_library()
    assert L.loopspec_sample_workspace_bytes(0, 1) == 0 and L.loopspec_sample_workspace_bytes(1000, 0) == 0
    need = L.loopspec_sample_workspace_bytes(1000, 4)
    assert need > 0 and _sample_rc(nbytes=need - 1) == B.EINVAL
