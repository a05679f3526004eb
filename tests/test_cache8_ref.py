"""The reference of a cache held in 8 bits by hand, and the host checks of the calls
that take one (nothing is enqueued on these paths, so no GPU is needed)."""
import ctypes
import os

import pytest
import torch

from tests import cache8_ref as c8
from tests.test_attention_abi import A, _kv, _rows, _seqs, ref


def test_reference_by_hand():
    # 448 2^-3 = 56 holds 50; the step there is 4: 50 is midway between 48 and 52, and 48's code is even
    codes, e = c8.hold(torch.tensor([[50.0, -50.0, 54.0, 0.5, 0.0]]), c8.E4M3)
    assert e.tolist() == [-3] and c8.worth(codes, e, c8.E4M3).tolist() == [[48.0, -48.0, 56.0, 0.5, 0.0]]
    # 127 2^0 holds 127 but not 127.5, whose row is counted in twos
    codes, e = c8.hold(torch.tensor([[127.0, 2.5, -3.5], [127.5, 1.0, 3.0]]), c8.I8)
    assert e.tolist() == [0, 1] and codes.tolist() == [[127, 2, -4], [64, 0, 2]]
    codes, e = c8.hold(torch.tensor([[0.0, 0.0], [torch.inf, 1.0], [torch.nan, 2.0]]), c8.I8)
    assert e.tolist() == [-96, -128, -128] and codes.tolist() == [[0, 0]] * 3
    codes, e = c8.hold(torch.tensor([[torch.inf, 448.0], [3e38, 1.0]]), c8.E4M3)
    assert codes[0].tolist() == [0x7F, 0x7E] and e.tolist() == [0, 119]
    assert c8.worth(codes, e, c8.E4M3)[1].tolist() == [448.0 * 2.0**119, 0.0]


def test_codes_round_trip():
    for t in (c8.E4M3, c8.I8):
        values, codes = c8.codes_of(t)
        assert torch.equal(codes.view(t).double(), values) and bool((values.diff() > 0).all())
        got, e = c8.hold(values[None] * 2.0**7, t)
        assert e.tolist() == [7] and torch.equal(got[0], codes)


@pytest.fixture(scope="module")
def L():
    from paper_2609_10264_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libmvk.so not built (run __graft_entry__.build())")
    return _lib


def _kv8(L, kind, k_exp=A, v_exp=A, kx_page=64, **kw):
    base = _kv(L, type=kind, **kw)
    return L.MvkKv8(*[getattr(base, f) for f, _ in L.MvkKv._fields_], k_exp, v_exp, kx_page, 16, 1, 64, 16, 1)


def test_struct_begins_with_the_plain_one(L):
    assert ctypes.sizeof(L.MvkKv8) == ctypes.sizeof(L.MvkKv) + 8 * 8
    assert all(getattr(L.MvkKv8, f).offset == getattr(L.MvkKv, f).offset for f, _ in L.MvkKv._fields_)


@pytest.mark.parametrize("kind", [4, 5])
def test_refusals(L, kind):
    lib = L.load()
    E, R = L.MVK_EINVAL, L.MVK_ERANGE
    bf, hf = _rows(L), _rows(L, type_=1)

    def read(kv=_kv8(L, kind), sq=_seqs(L), T=3, k=bf, v=_rows(L, data=A + (1 << 20))):
        p = [ref(x) if x is not None else None for x in (kv, sq, k, v)]
        return lib.mvk_cache_read(p[0], p[1], T, p[2], p[3], None)

    def append(kv=_kv8(L, kind), T=3, q=bf, out=_rows(L, data=A + (1 << 20)), k=_rows(L, data=A + (2 << 20))):
        return lib.mvk_rotary_append(ref(q), ref(k), ref(k), T, 8, 128, 128, 0, A, A, 10, 1.0, ref(out), ref(kv),
                                     ref(_seqs(L)), None)

    def attend(kv=_kv8(L, kind), T=3, q=bf):
        return lib.mvk_paged_attention(ref(q), T, 8, ref(kv), ref(_seqs(L)), 0.1, ref(_rows(L, data=A + (1 << 20))), 0.0,
                                       None, None, None, 0, 0, None)

    assert read(T=0) == append(T=0) == attend(T=0) == L.MVK_OK
    for call in (read, append, attend):
        assert call(kv=_kv8(L, kind, k_exp=None)) == E and call(kv=_kv8(L, kind, v_exp=None)) == E
        assert call(kv=_kv8(L, kind, kx_page=1 << 62)) == R and call(kv=_kv8(L, kind, K=None)) == E
        assert call(kv=_kv8(L, kind, page_size=24)) == E and call(kv=_kv8(L, kind, dim=513)) == R
    # queries over a cache held in 8 bits are bfloat16
    assert attend(q=hf) == E and attend(q=_rows(L, type_=kind)) == E
    assert append(out=_rows(L, type_=1, data=A + (1 << 20))) == E
    assert append(k=_rows(L, type_=kind, data=A + (2 << 20))) == E
    assert read(k=None, v=None) == E and read(kv=None) == E and read(sq=None) == E and read(sq=_seqs(L, q_start=None)) == E
    assert read(k=_rows(L, type_=3)) == E and read(k=_rows(L, type_=kind)) == E and read(v=bf) == E  # one memory for both
    assert read(T=1 << 31) == R and read(k=_rows(L, token=1 << 62)) == R
    other = _kv8(L, 9 - kind)
    assert lib.mvk_cache_evict(ref(_kv8(L, kind)), ref(_seqs(L)), A, 256, 64, 20, 4, 4, ref(other), A, 2, 2, None, 40, 20,
                               A, A, None) == E  # another type


def test_binding_refusals_without_a_gpu():
    import paper_2609_10264_amd as mvk
    pool = torch.zeros((2, 1, 16, 8), dtype=torch.int8)
    with pytest.raises(TypeError):
        mvk.KVCache(pool, pool, pool[..., 0], pool[..., 0]).struct()  # not on a GPU
    cache = mvk.KVCache.allocate(2, 1, 16, 8, dtype=torch.float8_e4m3fn, device="cpu")
    assert cache.k_exp.shape == (2, 1, 16) and cache.query_dtype == torch.bfloat16
    assert mvk.KVCache.allocate(2, 1, 16, 8, dtype=torch.float16, device="cpu").query_dtype == torch.float16
