"""What the paged-cache calls refuse, on the host and before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

from paper_2510_07651_b200 import api, build


@pytest.fixture(scope="module")
def L():
    build.build()
    return api.lib()


def _t(ptr=4096, dt=1, sb=2 * 16 * 128, sh=16 * 128, st=128):
    return api.obc_tensor(ptr, dt, sb, sh, st)


def _pages(**kw):
    dt = kw.pop("dt", api.OBC_BF16)
    base = dict(k=_t(dt=dt), v=_t(dt=dt), k_scale=None, v_scale=None, scale_stride_p=32, scale_stride_h=16, batch=2, n_kv_heads=2,
                head_dim=128, n_pages=10, page_size=16, max_pages=4, table=4096, table_stride_b=4, table_stride_h=0, lens=4096,
                lens_stride_b=1, lens_stride_h=0)
    if dt == api.OBC_E4M3:
        base.update(k_scale=4096, v_scale=8192)
    base.update(kw)
    return api.obc_pages(C.sizeof(api.obc_pages), *[base[n] for n, _ in api.obc_pages._fields_[1:]])


def _wp(**kw):
    base = dict(rows=4, src_tokens=4, new_lens=None, new_lens_stride_b=0, new_lens_stride_h=0, idx=None)
    base.update(kw)
    return api.obc_paged_write_params(C.sizeof(api.obc_paged_write_params), *[base[n] for n, _ in api.obc_paged_write_params._fields_[1:]])


def _ap(**kw):
    base = dict(n_q_heads=8, n_tokens=1, q_lens=None, scale=0.0, causal=1)
    base.update(kw)
    return api.obc_attention_params(C.sizeof(api.obc_attention_params), *[base[n] for n, _ in api.obc_attention_params._fields_[1:]])


BAD_PAGES = [
    (dict(head_dim=64), -3), (dict(batch=0), -2), (dict(n_kv_heads=0), -2), (dict(n_pages=0), -2), (dict(page_size=0), -2), (dict(page_size=12), -2),
    (dict(page_size=4), -2), (dict(max_pages=0), -2), (dict(max_pages=1 << 27), -2), (dict(batch=40000), -2), (dict(table=None), -1), (dict(lens=None), -1),
    (dict(table=4098), -4), (dict(lens=4097), -4), (dict(table_stride_b=-4), -2), (dict(lens_stride_h=-1), -2), (dict(k=_t(None)), -1), (dict(v=_t(None)), -1),
    (dict(k=_t(4104)), -4), (dict(v=_t(st=132)), -4), (dict(v=_t(st=64)), -2), (dict(k=_t(sb=-2048)), -2), (dict(v=_t(dt=0)), -3), (dict(k=_t(dt=3), v=_t(dt=3)), -3),
    (dict(k=_t(sh=0)), -2), (dict(k_scale=4096, v_scale=4096), -3), (dict(k=_t(sb=1 << 41)), -2), (dict(k=_t(sb=0)), -2), (dict(v=_t(sb=0)), -2),
    (dict(dt=2, k_scale=None), -1), (dict(dt=2, v_scale=None), -1), (dict(dt=2, k_scale=4100), -4), (dict(dt=2, scale_stride_p=20), -4),
    (dict(dt=2, scale_stride_h=-8), -2), (dict(dt=2, k=_t(dt=2, st=136)), -4),
]


@pytest.mark.parametrize("kw,want", BAD_PAGES)
def test_pages(L, kw, want):
    c, n = _pages(**kw), C.c_size_t(0)
    dt = kw.get("dt", 1)
    src = 0 if dt == 0 else 1
    assert L.obc_paged_write(C.byref(c), C.byref(_wp()), _t(dt=src), _t(dt=src), None) == want
    assert L.obc_paged_read(C.byref(c), 8, _t(dt=src), _t(dt=src), 0, None) == want
    assert L.obc_paged_attention_workspace(C.byref(c), C.byref(_ap()), C.byref(n)) == want
    assert L.obc_paged_attention(C.byref(c), C.byref(_ap()), _t(dt=src), _t(dt=src), 4096, 4096, 1 << 40, None) == want


def test_struct_sizes_and_missing_structs(L):
    n = C.c_size_t(0)
    c, a, w = _pages(), _ap(), _wp()
    assert L.obc_paged_write(None, C.byref(w), _t(), _t(), None) == -1 and L.obc_paged_write(C.byref(c), None, _t(), _t(), None) == -1
    assert L.obc_paged_read(None, 8, _t(), _t(), 0, None) == -1
    assert L.obc_paged_attention(C.byref(c), None, _t(), _t(), 4096, 4096, 1 << 40, None) == -1
    assert L.obc_paged_attention_workspace(C.byref(c), C.byref(a), None) == -1
    for s in (c, a, w):
        s.struct_size -= 8
    assert L.obc_paged_write(C.byref(_pages()), C.byref(w), _t(), _t(), None) == -3
    assert L.obc_paged_attention_workspace(C.byref(_pages()), C.byref(a), C.byref(n)) == -3
    assert L.obc_paged_read(C.byref(c), 8, _t(), _t(), 0, None) == -3


def test_write_and_read(L):
    c = _pages()
    w = lambda p, k=_t(), v=_t(): L.obc_paged_write(C.byref(c), C.byref(p), k, v, None)   # noqa: E731
    assert w(_wp(rows=0)) == -2 and w(_wp(src_tokens=0)) == -2 and w(_wp(rows=5)) == -2
    assert w(_wp(new_lens_stride_b=-1)) == -2 and w(_wp(new_lens=4097)) == -4 and w(_wp(idx=4098)) == -4
    assert w(_wp(), k=_t(None)) == -1 and w(_wp(), v=_t(4104)) == -4 and w(_wp(), k=_t(dt=0)) == -3 and w(_wp(), k=_t(dt=2), v=_t(dt=2)) == -3
    r = lambda n, k=_t(), v=_t(): L.obc_paged_read(C.byref(c), n, k, v, 0, None)          # noqa: E731
    assert r(0) == -2 and r(8, k=_t(None)) == -1 and r(8, k=_t(dt=0)) == -3 and r(8, k=_t(dt=2), v=_t(dt=2)) == -3 and r(8, v=_t(st=130)) == -4


def test_attention(L):
    c, n = _pages(), C.c_size_t(0)
    assert L.obc_paged_attention_workspace(C.byref(c), C.byref(_ap()), C.byref(n)) == 0 and n.value > 256 and n.value % 256 == 0
    f = lambda p=_ap(), q=_t(), o=_t(), lse=4096, ws=4096, size=n.value, c=c: L.obc_paged_attention(C.byref(c), C.byref(p), q, o, lse, ws, size, None)   # noqa: E731
    assert f(_ap(n_q_heads=7)) == -2 and f(_ap(n_q_heads=0)) == -2 and f(_ap(n_tokens=0)) == -2 and f(_ap(n_tokens=1 << 30)) == -2 and f(_ap(q_lens=4098)) == -4
    assert f(q=_t(None)) == -1 and f(o=_t(None)) == -1 and f(o=_t(4104)) == -4 and f(lse=4097) == -4
    assert f(o=_t(dt=0)) == -3 and f(q=_t(dt=0), o=_t(dt=0)) == -3 and f(c=_pages(dt=0)) == -3          # q in fp32 goes with fp32 pages alone
    assert f(ws=None) == -5 and f(size=n.value - 1) == -5 and f(ws=4224) == -4


def test_python_layer():
    import torch
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    cache = api.PagedCache(k, k, torch.zeros((1, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    q = torch.zeros((1, 2, 1, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA pages"):
        api.obc_paged_attention(q, cache)
    with pytest.raises(ValueError, match="CUDA pages"):
        api.obc_paged_write(cache, q, q)
    with pytest.raises(ValueError, match="CUDA pages"):
        api.obc_paged_read(cache)
    with pytest.raises(TypeError):
        api.obc_paged_read(cache, dtype=torch.float16)
    with pytest.raises(TypeError, match="torch.Tensor"):
        api.obc_paged_attention(q, cache._replace(k=None))
