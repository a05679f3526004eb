"""Host-side argument checks of the norm, activation and sampling calls, and the
references of their tests by hand (nothing is enqueued, so no GPU is needed)."""
import ctypes
import math
import os

import pytest
import torch

from tests import steps_ref
from tests.test_attention_abi import A, ref


@pytest.fixture(scope="module")
def L():
    from paper_2609_10264_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libmvk.so not built (run __graft_entry__.build())")
    return _lib


def _m(L, at=0, type_=0, stride=64):
    return L.MvkRows(A + at, type_, stride, 0)


FAR = 1 << 20


def test_struct_layouts(L):
    assert ctypes.sizeof(L.MvkNorm) == 8 + 8 + 4 + 4 + 8 and ctypes.sizeof(L.MvkSampling) == 3 * 8 + 8 + 4 * 8


def test_block_norm(L):
    lib = L.load()

    def call(x=_m(L), xs=1.0, res=_m(L, FAR), T=3, n=64, after=None, gate=None, scale=1.0, ro=_m(L, 2 * FAR),
             before=None, out=_m(L, 3 * FAR), os_=1.0):
        p = [ref(v) if v is not None else None for v in (x, res, after, gate, ro, before, out)]
        return lib.mvk_block_norm(p[0], xs, p[1], T, n, p[2], p[3], scale, p[4], p[5], p[6], os_, None)

    E, R = L.MVK_EINVAL, L.MVK_ERANGE
    w = L.MvkNorm(A + 4 * FAR, None, 2, 0, 1e-6)
    assert call(T=0) == L.MVK_OK and call(T=0, before=w, after=w) == L.MVK_OK
    assert call(x=None, res=None) == E and call(ro=None, out=None) == E and call(before=w, out=None) == E
    assert call(x=None, after=w) == E and call(x=None, gate=_m(L, 5 * FAR)) == E and call(n=0) == E
    assert call(scale=math.nan) == E and call(x=_m(L, type_=3), xs=math.inf) == E
    assert call(out=_m(L, 3 * FAR, type_=3), os_=0.0) == E and call(out=_m(L, 3 * FAR, type_=3), os_=math.nan) == E
    assert call(res=_m(L, FAR, type_=3)) == E and call(ro=_m(L, FAR, type_=3)) == E and call(gate=_m(L, 5 * FAR, type_=3)) == E
    assert call(x=_m(L, type_=4)) == E and call(x=_m(L, at=1)) == E
    for bad in (L.MvkNorm(A, None, 3, 0, 1e-6), L.MvkNorm(A, None, 2, 2, 1e-6), L.MvkNorm(A + 2, None, 2, 0, 1e-6),
                L.MvkNorm(A, None, 2, 0, -1.0), L.MvkNorm(A, None, 2, 0, math.nan)):
        assert call(before=bad) == E and call(after=bad) == E
    # outputs in the memory of inputs, of each other, of a norm's parameters; rows that meet
    assert call(ro=_m(L, FAR + 64)) == E and call(ro=_m(L)) == E and call(out=_m(L, FAR)) == E and call(out=_m(L, 2 * FAR)) == E
    assert call(out=_m(L, 64)) == E and call(out=_m(L, 5 * FAR), gate=_m(L, 5 * FAR)) == E
    assert call(out=_m(L, 4 * FAR), before=w) == E and call(ro=_m(L, 2 * FAR, stride=63)) == E and call(out=_m(L, 3 * FAR, stride=0)) == E
    assert call(out=_m(L, type_=1)) == E  # x's place in another type
    assert call(n=32769, x=None, res=_m(L, FAR, stride=1 << 20)) == R and call(T=1 << 31) == R
    assert call(x=_m(L, stride=1 << 62)) == R


def test_gated_activation(L):
    lib = L.load()

    def call(gate=_m(L), up=_m(L, FAR), T=3, n=64, act=0, s=1.0, out=_m(L, 2 * FAR), os_=1.0):
        p = [ref(v) if v is not None else None for v in (gate, up, out)]
        return lib.mvk_gated_activation(p[0], p[1], T, n, act, s, p[2], os_, None)

    E, R = L.MVK_EINVAL, L.MVK_ERANGE
    assert call(T=0) == L.MVK_OK
    assert call(gate=None) == E and call(up=None) == E and call(out=None) == E and call(n=0) == E
    assert call(act=4) == E and call(act=-1) == E and call(up=_m(L, FAR, type_=1)) == E and call(out=_m(L, 2 * FAR, stride=5)) == E
    f = _m(L, type_=3)
    assert call(gate=f, up=_m(L, FAR, type_=3), s=math.nan) == E and call(out=_m(L, 2 * FAR, type_=3), os_=-1.0) == E
    assert call(out=_m(L, 64)) == E and call(out=_m(L, FAR + 64)) == E and call(out=_m(L, type_=1)) == E
    assert call(n=1 << 31) == R and call(T=1 << 31) == R and call(gate=_m(L, stride=1 << 62)) == R


def test_sample_tokens(L):
    lib = L.load()

    def call(x=_m(L), R=3, n=64, fs=1.0, how=L.MvkSampling(1, 1, 0, 0), u=A + FAR, tok=A + 2 * FAR, probs=None):
        p = [ref(v) if v is not None else None for v in (x, how)]
        return lib.mvk_sample_tokens(p[0], R, n, fs, p[1], u, tok, probs, None)

    E, R = L.MVK_EINVAL, L.MVK_ERANGE
    assert call(R=0) == L.MVK_OK
    assert call(x=None) == E and call(how=None) == E and call(u=None) == E and call(tok=None) == E and call(n=0) == E
    assert call(x=_m(L, type_=3), fs=0.0) == E and call(x=_m(L, type_=3), fs=math.inf) == E and call(x=_m(L, type_=5)) == E
    assert call(tok=A + 8) == E and call(tok=A + FAR + 4) == E and call(probs=A + 2 * FAR + 8) == E and call(probs=A) == E
    for i in range(4):
        how = L.MvkSampling(1, 1, 0, 0, *[A + 3 * FAR if i == k else None for k in range(4)])
        assert call(how=how, tok=A + 3 * FAR) == E and call(how=how, probs=A + 3 * FAR) == E
    assert call(R=(1 << 24) + 1) == R and call(n=(1 << 24) + 1) == R and call(x=_m(L, stride=1 << 62)) == R


def test_reference_by_hand():
    x = torch.tensor([0.0, math.log(2.0), 0.0, math.log(4.0)], dtype=torch.float64)  # weights 1, 2, 1, 4 over 4
    at = lambda u, **kw: steps_ref.token(x, u, **{**dict(t=1.0, k=0, p=1.0, least=0.0), **kw})  # noqa: E731
    assert [at(u)[0] for u in (0.0, 0.124, 0.126, 0.374, 0.376, 0.499, 0.501, 0.99)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert at(0.99)[1] == pytest.approx(0.5)
    assert [at(u, k=2)[0] for u in (0.0, 0.33, 0.34)] == [1, 1, 3] and [at(u, k=3)[0] for u in (0.0, 0.15)] == [0, 1]
    assert at(0.0, p=0.49) == (3, 1.0) and at(0.0, p=0.51)[0] == 1 and at(0.0, p=0.76)[0] == 0
    assert at(0.0, least=0.49)[0] == 1 and at(0.0, least=0.51)[0] == 3 and at(0.9, t=0.0) == (3, 1.0)
    assert steps_ref.token(torch.full((3,), -math.inf), 0.5, 1.0, 0, 1.0, 0.0) == (-1, 0.0)


def test_binding_refusals_without_a_gpu():
    import paper_2609_10264_amd as mvk
    with pytest.raises(ValueError):
        mvk.Norm(kind="batch").struct(4, 0)
    with pytest.raises(TypeError):
        mvk.Norm(torch.ones(4)).struct(4, 0)
