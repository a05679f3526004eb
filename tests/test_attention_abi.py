"""Host-side argument checks of the client's attention calls (nothing is
enqueued on these paths, so no GPU is needed)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2609_10264_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libmvk.so not built (run __graft_entry__.build())")
    return _lib


ref = ctypes.byref
A = 0x10000  # an aligned address that nothing reads


def _rows(L, type_=0, token=4096, head=128, data=A):
    return L.MvkRows(data, type_, token, head)


def _kv(L, **kw):
    d = dict(K=A, V=A, type=0, pages=8, kv_heads=4, page_size=16, dim=128, k_page=4 * 16 * 128, k_head=16 * 128,
             k_entry=128, v_page=4 * 16 * 128, v_head=16 * 128, v_entry=128)
    d.update(kw)
    return L.MvkKv(*[d[f] for f, _ in L.MvkKv._fields_])


def _seqs(L, **kw):
    d = dict(table=A, table_stride=4, count=2, width=4, lens=A, q_start=A, max_new=1)
    d.update(kw)
    return L.MvkSeqs(*[d[f] for f, _ in L.MvkSeqs._fields_])


def test_struct_layouts_match_header(L):
    assert ctypes.sizeof(L.MvkRows) == 8 + 8 + 16
    assert ctypes.sizeof(L.MvkKv) == 16 + 5 * 4 + 4 + 6 * 8
    assert ctypes.sizeof(L.MvkSeqs) == 8 + 8 + 8 + 8 + 8 + 8


def test_rotary_table(L):
    f = L.load().mvk_rotary_table
    none, lin, base, parts = L.MVK_SCALE_NONE, L.MVK_SCALE_LINEAR, L.MVK_SCALE_BASE, L.MVK_SCALE_PARTS
    assert f(64, 0, 1e4, none, 1, 0, 1, 32, None, None) == L.MVK_OK  # no rows: no work
    for args in ((0, 8, 1e4, none, 1, 0, 1, 32), (7, 8, 1e4, none, 1, 0, 1, 32), (64, 8, 0.0, none, 1, 0, 1, 32),
                 (64, 8, float("nan"), none, 1, 0, 1, 32), (64, 8, 1e4, 4, 1, 0, 1, 32), (64, 8, 1e4, -1, 1, 0, 1, 32),
                 (64, 8, 1e4, lin, 0.5, 0, 1, 32), (2, 8, 1e4, base, 2, 0, 1, 32), (64, 8, 1e4, parts, 2, 0, 1, 32),
                 (64, 8, 1e4, parts, 2, 4096, 32, 1)):
        assert f(*args, A, None) == L.MVK_EINVAL, args
    assert f(64, 8, 1e4, none, 1, 0, 1, 32, None, None) == L.MVK_EINVAL
    assert f(514, 8, 1e4, none, 1, 0, 1, 32, A, None) == L.MVK_ERANGE
    assert f(64, 1 << 31, 1e4, none, 1, 0, 1, 32, A, None) == L.MVK_ERANGE


def test_rotary_append(L):
    lib = L.load()

    def call(q=_rows(L), k=_rows(L), v=_rows(L), T=3, heads=8, dim=128, rot=128, layout=0, pos=A, table=A, rows=10,
             scale=1.0, out=_rows(L), kv=_kv(L), sq=_seqs(L)):
        p = [ref(x) if x is not None else None for x in (q, k, v, out, kv, sq)]
        return lib.mvk_rotary_append(p[0], p[1], p[2], T, heads, dim, rot, layout, pos, table, rows, scale, p[3], p[4],
                                     p[5], None)

    out = _rows(L, data=A + 4096)
    assert call(T=0, out=out) == L.MVK_OK
    E = L.MVK_EINVAL
    assert call(q=None) == E and call(out=None) == E and call(k=None) == E and call(v=None) == E
    assert call(kv=None) == E and call(sq=None) == E
    assert call(q=None, k=None, v=None, out=None, kv=None, sq=None) == E
    assert call(layout=2) == E and call(rot=63) == E and call(rot=130) == E and call(dim=0) == E
    assert call(pos=None) == E and call(table=None) == E and call(rows=0) == E and call(heads=0) == E
    assert call(out=_rows(L, type_=L.MVK_TYPE_FIELD)) == E  # floats only
    assert call(out=_rows(L, type_=1)) == E  # not the cache's type
    assert call(out=_rows(L, token=4104)) == E  # in place with other strides
    assert call(k=_rows(L, type_=2), v=_rows(L, type_=2)) == E and call(v=_rows(L, type_=1)) == E
    assert call(dim=64, rot=64) == E  # another dim than the cache's
    assert call(q=_rows(L, type_=9)) == E and call(q=_rows(L, data=A + 1)) == E and call(q=_rows(L, data=None)) == E
    assert call(kv=_kv(L, page_size=24)) == E and call(kv=_kv(L, pages=0)) == E and call(kv=_kv(L, type=3)) == E
    f = _rows(L, type_=3)
    assert call(q=f, k=f, v=f, scale=float("inf")) == E
    R = L.MVK_ERANGE
    assert call(dim=520, rot=64, kv=None, sq=None, k=None, v=None) == R
    assert call(T=1 << 31) == R and call(heads=65536) == R
    assert call(q=_rows(L, token=1 << 62)) == R
    assert call(kv=_kv(L, k_page=1 << 62)) == R and call(kv=_kv(L, v_entry=1 << 60)) == R
    assert call(sq=_seqs(L, width=1 << 28, table_stride=1 << 28)) == R and call(sq=_seqs(L, count=65536)) == R


def test_paged_attention(L):
    lib = L.load()

    def call(q=_rows(L), T=3, heads=8, kv=_kv(L), sq=_seqs(L), scale=0.1, out=_rows(L), fs=1.0, lse=None, wi=None,
             wo=None, ws=256, wh=64):
        p = [ref(x) if x is not None else None for x in (q, kv, sq, out)]
        return lib.mvk_paged_attention(p[0], T, heads, p[1], p[2], scale, p[3], fs, lse, wi, wo, ws, wh, None)

    assert call(T=0) == L.MVK_OK
    E, R = L.MVK_EINVAL, L.MVK_ERANGE
    assert call(q=None) == E and call(kv=None) == E and call(sq=None) == E and call(out=None) == E
    assert call(heads=0) == E and call(heads=6) == E and call(scale=float("nan")) == E
    assert call(q=_rows(L, type_=1)) == E and call(q=_rows(L, type_=3)) == E
    assert call(out=_rows(L, type_=3), fs=0.0) == E and call(out=_rows(L, type_=3), fs=float("inf")) == E
    assert call(wi=A) == E and call(wo=A, wh=63) == E and call(wo=A, ws=63) == E
    assert call(sq=_seqs(L, q_start=None)) == E and call(sq=_seqs(L, lens=None)) == E and call(sq=_seqs(L, table=None)) == E
    assert call(sq=_seqs(L, count=0)) == E and call(sq=_seqs(L, width=0)) == E and call(sq=_seqs(L, table_stride=3)) == E
    assert call(kv=_kv(L, K=None)) == E and call(kv=_kv(L, V=A + 1)) == E and call(kv=_kv(L, page_size=0)) == E
    assert call(T=1 << 29, heads=8) == R and call(kv=_kv(L, dim=513)) == R
    assert call(wo=A, ws=1 << 62) == R and call(out=_rows(L, head=1 << 61)) == R
    assert call(sq=_seqs(L, table_stride=1 << 61)) == R


def test_cache_evict(L):
    lib = L.load()

    def call(src=_kv(L), sq=_seqs(L, q_start=None), w=A, ws=256, wh=64, budget=20, recent=4, sinks=4, dst=_kv(L), dt=A,
             ds=2, dw=2, wo=None, os_=40, oh=20, kept=A, lens=A):
        p = [ref(x) if x is not None else None for x in (src, sq, dst)]
        return lib.mvk_cache_evict(p[0], p[1], w, ws, wh, budget, recent, sinks, p[2], dt, ds, dw, wo, os_, oh, kept,
                                   lens, None)

    E, R = L.MVK_EINVAL, L.MVK_ERANGE
    assert call(src=None) == E and call(dst=None) == E and call(sq=None) == E and call(w=None) == E
    assert call(dt=None) == E and call(kept=None) == E and call(lens=None) == E
    assert call(budget=0, recent=0, sinks=0) == E and call(recent=17) == E
    assert call(recent=0xFFFFFFFF, sinks=0xFFFFFFFF) == E  # the sum is taken in 64 bits
    assert call(dst=_kv(L, type=1)) == E and call(dst=_kv(L, dim=64)) == E and call(dst=_kv(L, kv_heads=2)) == E
    assert call(wh=63) == E and call(ws=63) == E and call(wo=A, oh=19) == E and call(wo=A, os_=19) == E
    assert call(dw=1) == E and call(ds=1) == E and call(dw=0) == E
    assert call(budget=1 << 31, dst=_kv(L, page_size=1 << 20), dw=2) == R
    assert call(ws=1 << 62) == R and call(src=_kv(L, k_head=1 << 61)) == R
