"""Which kernels the attention calls launch, with which grids, up to the sizes that
the header allows (the library's host side; nothing is computed)."""
from tests.test_host_dispatch import host  # noqa: F401

STRUCTS = """
def rows(data, type_, heads, dim): return L.MvkRows(data, type_, heads * dim, dim)
def kv(heads, dim, type_=0, page=16, pages=8):
    return L.MvkKv(ptr(), ptr(), type_, pages, heads, page, dim, *((heads * page * dim, page * dim, dim) * 2))
def seqs(count, width, max_new): return L.MvkSeqs(ptr(), width, count, width, ptr(), ptr(), max_new)
def grids():
    g, out = (ctypes.c_uint32 * 3)(), []
    for i in range(rec.rec_count()):
        rec.rec_grid(i, g)
        out.append([rec.rec_name(i).decode().replace("void ", "").replace("mvk::(anonymous namespace)::", "").split("<")[0],
                    g[0], g[0] * g[2] < 2**32])
    return out
def attend(T, heads, kv_heads, dim, type_=0, count=1, width=4, page=16, max_new=None, w=None):
    cache, sq = kv(kv_heads, dim, type_, page), seqs(count, width, T if max_new is None else max_new)
    cap = width * page
    q, out = rows(ptr(), type_, heads, dim), rows(ptr(), type_, heads, dim)
    call = lambda: lib.mvk_paged_attention(ref(q), T, heads, ref(cache), ref(sq), 0.1, ref(out), 1.0, None, None, w,  # noqa
                                           kv_heads * cap, cap, None)
    call()  # (the workspace's own launches)
    rec.rec_reset()
    return [call(), grids()]
"""


def test_rows_of_the_general_kernel(host):  # noqa: F811
    """Up to 2^31 - 1 rows in launches of fewer than 2^32 threads."""
    out = host(STRUCTS + """
for T, heads in ((3, 5), (2**20, 16), (2**20, 64), (2**25, 63), (2**31 - 1, 1)):
    result[f"{T} x {heads}"] = attend(T, heads, 1, 4, type_=2)
""")
    for name, (st, launches) in out.items():
        assert st == 0 and [x[0] for x in launches] == ["attend_any"] and launches[0][2], (name, launches)
    assert out["3 x 5"][1][0][1] == 4


def test_rows_of_the_eviction(host):  # noqa: F811
    """Up to 2^31 - 1 kept entries in launches of fewer than 2^32 threads."""
    out = host(STRUCTS + """
def evict(n, dim, page):
    K, V = ptr() + 2, ptr() + 2  # (no 16-byte rows)
    width = -(-n // page)
    src = L.MvkKv(K, V, 0, 8, 1, page, dim, *((page * dim, page * dim, dim) * 2))
    sq = seqs(1, width, 0)
    rec.rec_reset()
    return [lib.mvk_cache_evict(ref(src), ref(sq), ptr(), n, n, n, 0, 0, ref(src), ptr(), width, width, None, 0, 0,
                                ptr(), ptr(), None), grids()]
for n, dim in ((100, 512), (2**25, 512), (2**26 + 1, 512), (2**30, 300), (2**31 - 2**20, 1)):
    result[f"{n} of {dim}"] = evict(n, dim, 2**20 if n > 100 else 16)
""")
    for name, (st, launches) in out.items():
        assert st == 0 and [x[0].split("(")[0] for x in launches] == ["evict_select", "evict_copy"], (name, launches)
        assert all(x[2] for x in launches), (name, launches)
