"""Refusals of the full-attention calls: all are decided on the host, before any HIP call."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_11231_amd", "liblkv.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="liblkv.so not built")
torch = pytest.importorskip("torch")

from paper_2608_11231_amd import lkv  # noqa: E402

NULL, SHAPE, DTYPE, ALIGN, UNSUPPORTED = 1, 2, 3, 4, 5
P = 0x1000  # an aligned address that no refused call follows


def _attn(**kw):
    d = dict(h_q=8, h_kv=2, d=128, page=64, io_dtype=1, cache_dtype=1, scale=0.1)
    d.update(kw)
    return lkv.Attn(**d)


def _pages(**kw):
    d = dict(k=P, v=P, k_exp=None, v_exp=None, n_page=4, max_pages=2, table=P, len=P)
    d.update(kw)
    return lkv.Pages(**d)


def _prefill(a, n_seq=1, n_tok=4, cu=P, q=P, qs=1024, k=P, ks=256, v=P, vs=256, o=P):
    return lkv.load().lkv_attn_prefill(a, cu, n_seq, n_tok, q, qs, k, ks, v, vs, o, None)


def _paged(a, pg, n_req=1, n_tok=4, cu=P, pos=None, q=P, qs=1024, o=P, ws=P, ws_bytes=1 << 30):
    return lkv.load().lkv_attn_paged(a, pg, cu, n_req, n_tok, pos, q, qs, o, ws, ws_bytes, None)


def _moves(a, pg, n_req=1, n_tok=4, cu=P, k=P, ks=256, v=P, vs=256):
    st = {f(a, pg, cu, n_req, n_tok, None, k, ks, v, vs, None) for f in (lkv.load().lkv_kv_write, lkv.load().lkv_kv_read)}
    assert len(st) == 1
    return st.pop()


BAD_LAYERS = [(dict(h_kv=3), SHAPE), (dict(h_q=0), SHAPE), (dict(h_kv=0), SHAPE), (dict(scale=0.0), SHAPE),
              (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
              (dict(io_dtype=2), DTYPE), (dict(io_dtype=7), DTYPE), (dict(cache_dtype=0), DTYPE), (dict(cache_dtype=9), DTYPE),
              (dict(io_dtype=0, cache_dtype=2), DTYPE), (dict(io_dtype=0, cache_dtype=1), DTYPE),
              (dict(d=96), UNSUPPORTED), (dict(d=512), UNSUPPORTED), (dict(io_dtype=0, cache_dtype=0, d=256), UNSUPPORTED),
              (dict(page=0), SHAPE), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=2048), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD_LAYERS)
def test_layers(bad, status):
    a = _attn(**bad)
    n = ctypes.c_size_t(0)
    assert _prefill(a) == _paged(a, _pages()) == _moves(a, _pages()) == status
    assert lkv.load().lkv_attn_paged_workspace(a, 1, 4, 2, ctypes.byref(n)) == status


def test_prefill_arguments():
    a = _attn()
    assert lkv.load().lkv_attn_prefill(None, P, 1, 4, P, 1024, P, 256, P, 256, P, None) == NULL
    assert _prefill(a, n_seq=0) == _prefill(a, n_tok=0) == 0
    assert _prefill(a, n_seq=-1) == _prefill(a, n_tok=-1) == _prefill(a, n_tok=1 << 31) == SHAPE
    assert [_prefill(a, **{x: None}) for x in ("cu", "q", "k", "v", "o")] == [NULL] * 5
    assert [_prefill(a, **{x: P + 8}) for x in ("q", "k", "v", "o")] == [ALIGN] * 4
    assert [_prefill(a, **{x: 128}) for x in ("qs", "ks", "vs")] == [SHAPE] * 3  # rows would overlap
    assert [_prefill(a, **{x: 1028}) for x in ("qs", "ks", "vs")] == [ALIGN] * 3
    assert [_prefill(a, **{x: (1 << 22) + 8}) for x in ("qs", "ks", "vs")] == [UNSUPPORTED] * 3


def test_paged_arguments():
    a = _attn()
    assert _paged(a, None) == _moves(a, None) == NULL
    for f in (_paged, _moves):
        assert f(a, _pages(), n_req=0) == f(a, _pages(), n_tok=0) == 0
        assert f(a, _pages(), n_req=-1) == f(a, _pages(), n_tok=-1) == SHAPE
        assert f(a, _pages(), cu=None) == NULL
        for bad, status in ((dict(n_page=-1), SHAPE), (dict(max_pages=-1), SHAPE), (dict(max_pages=1 << 26), SHAPE),
                            (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL), (dict(len=None), NULL),
                            (dict(k=P + 8), ALIGN), (dict(v=P + 8), ALIGN)):
            assert f(a, _pages(**bad), n_tok=4) == status, bad
        assert f(_attn(cache_dtype=2), _pages(k_exp=P)) == NULL  # v_exp missing
    assert _paged(a, _pages(), q=None) == _paged(a, _pages(), o=None) == NULL
    assert _paged(a, _pages(), q=P + 2) == _paged(a, _pages(), o=P + 2) == _paged(a, _pages(), qs=1028) == ALIGN
    assert _paged(a, _pages(), qs=512) == SHAPE
    assert _moves(a, _pages(), ks=248) == _moves(a, _pages(), vs=248) == SHAPE


def test_too_many_workgroups():
    """Launches past 2^24 workgroups are refused, on whichever grid is the large one."""
    a, one = _attn(), _attn(h_q=1, h_kv=1)
    assert _moves(one, _pages(), n_tok=1 << 26) == SHAPE
    assert _prefill(one, n_tok=(1 << 31) - 1, qs=128, ks=128, vs=128) == SHAPE
    assert _prefill(one, n_seq=1 << 24, n_tok=1, qs=128, ks=128, vs=128) == SHAPE
    assert _paged(a, _pages(max_pages=1), n_req=1 << 23, n_tok=1 << 23) == SHAPE
    assert _paged(one, _pages(max_pages=1), n_req=1 << 26, n_tok=1 << 30, qs=128) == SHAPE


@pytest.mark.parametrize("bad", [(0, 2, 128), (8, 0, 128), (8, 2, 0), (8, 2, -64)], ids=str)
def test_make_attn_of_nothing(bad):
    with pytest.raises(ValueError):
        lkv.make_attn(*bad)


def test_workspace():
    a = _attn()
    need = lkv.attn_paged_workspace(a, 1, 4, 512)  # one request, a long context: split
    assert need > 0
    assert _paged(a, _pages(max_pages=512), ws=None) == NULL
    assert _paged(a, _pages(max_pages=512), ws=P + 16) == ALIGN
    assert _paged(a, _pages(max_pages=512), ws_bytes=need - 1) == SHAPE
    assert lkv.attn_paged_workspace(a, 0, 0, 512) == 0
    assert lkv.attn_paged_workspace(a, 4096, 4096, 512) == 0  # the requests fill the GPU
    n = ctypes.c_size_t(0)
    f = lkv.load().lkv_attn_paged_workspace
    assert f(a, 1, 4, 512, None) == NULL and f(a, -1, 4, 512, ctypes.byref(n)) == SHAPE
    assert f(a, 1, 4, -1, ctypes.byref(n)) == f(a, 1, 4, 1 << 26, ctypes.byref(n)) == SHAPE


def test_binding_checks():
    with pytest.raises(ValueError):
        lkv.make_attn(8, 2, 128, io_dtype=torch.float16)
    a = lkv.make_attn(8, 2, 128)
    assert abs(a.scale - 128 ** -0.5) < 1e-8 and a.cache_dtype == a.io_dtype == lkv.BF16
    x = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    bad = [x.float(), x[:3], x[:, :4], x[:, :, :64], x.reshape(4, 1024), x.transpose(0, 1).contiguous().transpose(0, 1)]
    for t in bad:
        with pytest.raises(ValueError):
            lkv._rows(a, t, 4, 8, "q")
    pages = torch.zeros((3, 2, 64, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lkv.make_pages(a, pages.float(), pages, None, None)
    with pytest.raises(ValueError):
        lkv.make_pages(a, pages, pages, None, None, k_exp=pages)
