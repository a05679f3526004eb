"""Outputs in an input's memory that a call cannot write without changing its own
results are refused, and views of one buffer that do not meet are taken (the
library's host side; nothing is computed)."""
from tests.test_host_dispatch import host  # noqa: F401

STRUCTS = """
def rows(data, type_=0, token=1024, head=128): return L.MvkRows(data, type_, token, head)
def kv(heads=4, dim=128):
    K, V = ptr(), ptr()
    return L.MvkKv(K, V, 0, 8, heads, 16, dim, heads * 16 * dim, 16 * dim, dim, heads * 16 * dim, 16 * dim, dim)
def seqs(count=2): return L.MvkSeqs(ptr(), 4, count, 4, ptr(), ptr(), 1)
"""


def test_eviction_weights(host):  # noqa: F811
    out = host(STRUCTS + """
w = ptr()
def call(wo, o_seq=256, o_head=64, w_seq=256, w_head=64):
    src, dst, sq = kv(), kv(), seqs()
    rec.rec_reset()
    st = lib.mvk_cache_evict(ref(src), ref(sq), w, w_seq, w_head, 20, 4, 4, ref(dst), ptr(), 2, 2, wo, o_seq, o_head,
                             ptr(), ptr(), None)
    return [st, rec.rec_count()]
result["itself"] = call(w)
result["a row on"] = call(w + 4 * 64)
result["one float before its end"] = call(w + 4 * (2 * 256 - 1))
result["behind it"] = call(w + 4 * 2 * 256)
result["the last float of w_out"] = call(w - 4 * (256 + 3 * 64 + 19))
result["before it"] = call(w - 4 * (256 + 3 * 64 + 20))
# views of one buffer, count x 2 x heads x 64 and count x heads x 2 x 64
result["seqs interleaved"] = call(w + 4 * 256, o_seq=512, w_seq=512)
result["heads interleaved"] = call(w + 4 * 64, o_seq=512, o_head=128, w_seq=512, w_head=128)
result["heads interleaved, a float short"] = call(w + 4 * 63, o_seq=512, o_head=128, w_seq=512, w_head=128)
result["other strides"] = call(w + 4 * 64, o_seq=1024, o_head=128, w_seq=512, w_head=128)
""")
    refused, done = [-1, 0], [0, 2]  # (MVK_EINVAL)
    assert out == {"itself": refused, "a row on": refused, "one float before its end": refused, "behind it": done,
                   "the last float of w_out": refused, "before it": done, "seqs interleaved": done,
                   "heads interleaved": done, "heads interleaved, a float short": refused, "other strides": refused}


def test_attention_in_the_memory_of_its_queries(host):  # noqa: F811
    out = host(STRUCTS + """
q = ptr()
def call(o, type_=0, token=1024, head=128, wo=None, wi=None, q_token=1024, q_head=128, dim=128, heads=8):
    cache, sq = kv(dim=dim), seqs()
    rec.rec_reset()
    st = lib.mvk_paged_attention(ref(rows(q, 0, q_token, q_head)), 3, heads, ref(cache), ref(sq), 0.1,
                                 ref(rows(o, type_, token, head)), 1.0, None, wi, wo, 256, 64, None)
    return [st, rec.rec_count() > 0]
call(ptr(), wo=ptr())  # (the workspace's own launches)
w = ptr()
for dim in (128, 100):  # both kernels
    r = result[str(dim)] = {}
    r["apart"] = call(ptr(), dim=dim), call(ptr(), dim=dim, wo=w)
    r["itself"] = call(q, dim=dim), call(q, dim=dim, wo=w)
    r["another type"] = call(q, type_=1, dim=dim), call(q, type_=2, dim=dim)
    r["other strides"] = call(q, token=2048, dim=dim), call(q, head=256, token=2048, dim=dim)
    r["a head on"] = call(q + 256, dim=dim), call(q + 256, dim=dim, wo=w)
    r["a token before"] = call(q - 2048, dim=dim), call(q - 2048, dim=dim, wo=w)
    # q and out as parts of one row of heads, and as halves of one head
    r["beside"] = [call(q + 2048, token=2048, q_token=2048, dim=dim, wo=x) for x in (None, w)]
    r["beside, a head short"] = [call(q + 2048 - 256, token=2048, q_token=2048, dim=dim, wo=x) for x in (None, w)]
    r["halves"] = [call(q + 256, token=2048, head=256, q_token=2048, q_head=256, dim=dim, wo=x) for x in (None, w)]
result["w"] = [call(ptr(), wo=w, wi=x) for x in (w, None, ptr(), w + 4, w + 4 * 64, w - 4 * 64, w + 4 * 512)]
""")
    no, yes = [-1, False], [0, True]
    for dim in ("128", "100"):
        assert out[dim] == {"apart": [yes, yes], "itself": [yes, no], "another type": [no, no],
                            "other strides": [no, no], "a head on": [no, no], "a token before": [no, no],
                            "beside": [yes, yes], "beside, a head short": [no, no], "halves": [yes, yes]}, dim
    assert out["w"] == [yes, yes, yes, no, no, no, yes]


def test_strides_that_no_second_row_uses(host):  # noqa: F811
    """One token, or one head: its stride says nothing, whatever a view happens to have."""
    out = host(STRUCTS + """
def call(T, heads, q, q_token, q_head, o, token, head):
    cache, sq = kv(heads=1), seqs()
    rec.rec_reset()
    w = ptr()
    st = lib.mvk_paged_attention(ref(rows(q, 0, q_token, q_head)), T, heads, ref(cache), ref(sq), 0.1,
                                 ref(rows(o, 0, token, head)), 1.0, None, None, w, 64, 64, None)
    return st
call(1, 1, ptr(), 128, 128, ptr(), 128, 128)
q = ptr()
# q and out as the halves of each token's row of two heads
result["one head"] = [call(3, 1, q, 256, x, q + 256, 256, y) for x, y in ((128, 128), (0, 256), (256, 128), (1 << 20, 0))]
result["one head, meeting"] = [call(3, 1, q, 256, x, q + 254, 256, y) for x, y in ((128, 128), (1 << 20, 0))]
# of one token, every second head
result["one token"] = [call(1, 4, q, x, 256, q + 256, y, 256) for x, y in ((1024, 1024), (0, 1 << 30), (128, 512))]
result["one token, meeting"] = [call(1, 4, q, x, 256, q + 512, y, 256) for x, y in ((1024, 1024), (128, 512))]
result["one row"] = [call(1, 1, q, 7, 9, q + x, 11, 13) for x in (256, 254, -254, -256)]
""")
    assert out == {"one head": [0] * 4, "one head, meeting": [-1] * 2, "one token": [0] * 3,
                   "one token, meeting": [-1] * 2, "one row": [0, -1, -1, 0]}


def test_rotary_in_the_memory_of_its_inputs(host):  # noqa: F811
    out = host(STRUCTS + """
def call(q, k, v, o, type_=0, o_type=0, token=1024, q_token=1024, kv_heads=4, kv_head=128):
    cache, sq = kv(heads=kv_heads), seqs()
    rec.rec_reset()
    st = lib.mvk_rotary_append(ref(rows(q, type_, q_token)), ref(rows(k, type_, q_token, kv_head)),
                               ref(rows(v, type_, q_token, kv_head)), 3, 8, 128, 128, 0, ptr(), ptr(), 100, 1.0,
                               ref(rows(o, o_type, token)), ref(cache), ref(sq), None)
    return [st, rec.rec_count() > 0]
q, k, v = ptr(), ptr(), ptr()
result["apart"] = call(q, k, v, ptr())
result["itself"] = call(q, k, v, q)
result["itself, another type"] = call(q, k, v, q, type_=2)
result["itself, other strides"] = call(q, k, v, q, token=2048)
result["shifted"] = [call(q, k, v, q + x) for x in (256, -2048, 2 * 3 * 1024 - 2)]
result["k, v"] = [call(q, k, v, k), call(q, k, v, v - 2048)]
# q, k and v parts of one row (8 + 4 + 4 heads of 128), q rotated in place
result["one row"] = call(q, q + 2048, q + 3072, q, token=2048, q_token=2048)
result["one row of one kv head"] = [call(q, q + 2048, q + 2304, q, token=1280, q_token=1280, kv_heads=1, kv_head=x) for x in (128, 1280)]
result["a row into its keys"] = call(q, q + 2048, q + 3072, q + 2048, token=2048, q_token=2048)
""")
    no, yes = [-1, False], [0, True]
    assert out == {"apart": yes, "itself": yes, "itself, another type": no, "itself, other strides": no,
                   "shifted": [no, no, no], "k, v": [no, no], "one row": yes, "one row of one kv head": [yes, yes],
                   "a row into its keys": no}


def test_parts_of_one_row_with_head_strides_of_their_own(host):  # noqa: F811
    """Queries one head after another, then keys and values by turns, in one row of a
    token: the queries rotated in place meet neither; and shifted ones do."""
    out = host(STRUCTS + """
def call(q, k, v, o, T=3, heads=8, kv_heads=4):
    width, cache, sq = (heads + 2 * kv_heads) * 128, kv(heads=kv_heads), seqs()
    rec.rec_reset()
    return lib.mvk_rotary_append(ref(rows(q, 0, width)), ref(rows(k, 0, width, 256)), ref(rows(v, 0, width, 256)), T,
                                 heads, 128, 128, 0, ptr(), ptr(), 100, 1.0, ref(rows(o, 0, width)), ref(cache),
                                 ref(sq), None)
x = ptr()
result["in place"] = [call(x, x + 2 * 128 * h, x + 2 * 128 * (h + 1), x, T, h, g) for T, h, g in ((3, 8, 4), (1, 8, 4), (2000, 64, 8), (3, 4, 1))]
y = ptr()
result["into the keys"] = [call(y, x, x + 256, x + 256 * i) for i in (-1, 0, 1, 5)]
result["of the next token"] = [call(y, x, x + 256, x + 256 * i) for i in (8, 9, 15)]
result["beside the keys"] = [call(y, x + 2 * 128 * 8, x + 2 * 128 * 9, x)]
result["many heads"] = [call(x, x + 2 * 128 * 512, x + 2 * 128 * 513, x, 3, 512, 256)]
""")
    assert out == {"in place": [0] * 4, "into the keys": [-1] * 4, "of the next token": [0, -1, -1],
                   "beside the keys": [0], "many heads": [0]}
