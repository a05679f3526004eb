"""Attention whose result takes the place of its queries (mvk_paged_attention)."""
import pytest
import torch

from tests.test_gpu_attention import BF, F32, HF, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# tiles of several workgroups, of both forms, and the general path
@pytest.mark.parametrize("lens,new,dim,dtype", [([5000, 70], [1, 1], 128, BF), ([5003, 700, 64], [150, 130, 64], 64, HF),
                                                ([3000, 90], [1, 1], 100, BF), ([300, 90], [40, 90], 64, F32)])
def test_out_is_q(lens, new, dim, dtype):
    import paper_2609_10264_amd as mvk
    pr = Problem(lens, new, 8, 2, dim, dtype=dtype).device()
    want = mvk.paged_attention(pr.dq, pr.cache, pr.seqs)
    q = pr.dq.clone()
    assert mvk.paged_attention(q, pr.cache, pr.seqs, out=q) is q
    assert torch.equal(q, want)


def test_not_where_the_queries_are_read_again():
    import paper_2609_10264_amd as mvk
    pr = Problem([300, 90], [40, 1], 8, 2, 64).device()
    q, w = pr.dq.clone(), torch.zeros((2, 2, pr.cap), device="cuda")
    with pytest.raises(mvk.MvkError):
        mvk.paged_attention(q, pr.cache, pr.seqs, out=q, weights=w)
    assert torch.equal(q, pr.dq) and not bool(w.any())
    # queries and result side by side in one buffer are apart
    both = torch.zeros((41, 16, 64), dtype=BF, device="cuda")
    both[:, :8] = pr.dq
    mvk.paged_attention(both[:, :8], pr.cache, pr.seqs, out=both[:, 8:], weights=w)
    w2 = torch.zeros_like(w)
    want = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, weights_out=w2)
    assert torch.equal(both[:, :8], pr.dq) and torch.equal(both[:, 8:], want) and torch.equal(w, w2)
