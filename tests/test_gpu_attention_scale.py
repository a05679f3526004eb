"""Scales of the scores: their sign, zero and the smallest, in the result, the sums
and the collected weights alike; and the hint of new tokens, which changes no result."""
import pytest
import torch

from tests.test_gpu_attention import BF, F32, HF, Problem, _within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _check(pr, scale=None, hint=None):
    import paper_2609_10264_amd as mvk
    print(f"attention lens={pr.lens} new={pr.new} q={tuple(pr.q.shape)} scale={scale} hint={hint}", flush=True)
    pr.device()
    if hint is not None:
        pr.seqs.max_new = hint
    T, H, _ = pr.q.shape
    lse = torch.full((T, H), 123.0, device="cuda")
    w = torch.full((len(pr.lens), pr.K.shape[1], pr.cap), -5.0, device="cuda")
    out = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, scale=scale, lse=lse, weights_out=w)
    torch.cuda.synchronize()
    r = pr.reference(scale=scale)
    _within(out, r.o, r.o_err, "o")
    _within(lse, r.lse, r.lse_err, "lse")
    for s, n in enumerate(pr.lens):
        _within(w[s, :, :n], r.w[s, :, :n], r.w_err[s, :, :n], f"w of sequence {s}")


KINDS = [(128, BF), (80, HF), (33, BF), (64, F32)]


@pytest.mark.parametrize("dim,dtype", KINDS)
@pytest.mark.parametrize("scale", [0.5, 0.01, 0.0, -0.0, -0.1])
def test_scale(scale, dim, dtype):
    _check(Problem([70, 33, 300, 0], [20, 33, 1, 1], 4, 2, dim, dtype=dtype), scale)


# scores of the size of one, from values whose products nearly fill 32 bits
@pytest.mark.parametrize("dim,dtype", [(128, BF), (33, BF), (64, F32)])
@pytest.mark.parametrize("size,scale", [(2.0**50, 2.0**-102), (2.0**57, 2.0**-116), (2.0**57, -2.0**-116)])
def test_smallest_scales(size, scale, dim, dtype):
    pr = Problem([70, 33, 300], [20, 33, 1], 4, 2, dim, dtype=dtype)
    pr.q, pr.K = (pr.q * size).to(dtype), (pr.K * size).to(dtype)
    _check(pr, scale)


# few new tokens announced where there are many, and many where there are few
@pytest.mark.parametrize("dim,dtype", KINDS)
@pytest.mark.parametrize("hint", [0, 1, 5, 10**6, None])
@pytest.mark.parametrize("lens,new,heads,kv_heads", [([500, 130, 64, 9], [300, 130, 1, 5], 8, 2), ([700, 65, 33, 2], [1, 1, 1, 1], 6, 6),
                                                     ([2500], [90], 14, 1)])
def test_the_hint_changes_no_result(hint, lens, new, heads, kv_heads, dim, dtype):
    pr = Problem(lens, new, heads, kv_heads, dim, dtype=dtype)
    _check(pr, hint=10**6 if hint is None else hint)
    if hint is None:
        pr.seqs.max_new = None
        import paper_2609_10264_amd as mvk
        r = pr.reference()
        _within(mvk.paged_attention(pr.dq, pr.cache, pr.seqs), r.o, r.o_err, "no hint")
