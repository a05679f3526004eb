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
        name = rec.rec_name(i).decode()  # (not every type's name is known to the demangler)
        kernels = ("attend_any", "attend_tile", "weights_any", "weights_tile", "evict_select", "evict_copy")
        out.append([next((k for k in kernels if k in name), name), g[0], g[0] * g[2] < 2**32])
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
        assert st == 0 and [x[0] for x in launches] == ["evict_select", "evict_copy"], (name, launches)
        assert all(x[2] for x in launches), (name, launches)


def test_large_batches_run_on_the_matrix_cores(host):  # noqa: F811
    """The tile kernels take what their counts hold, by the units that sequences can have
    in a table of that width, not by all token rows over all token rows."""
    out = host(STRUCTS + """
w = ptr()
for name, kw in {
    "64 prompts of 8192": dict(T=64 * 8192, count=64, width=128, page=64, max_new=8192),
    "a prompt of 200000": dict(T=200000, width=3125, page=64),
    "a prompt of 262144": dict(T=262144, heads=32, kv_heads=32, width=4096, page=64),
    "few prompts, wide table": dict(T=65536, count=8, width=1 << 14, page=64, max_new=8192),
    "65535 single tokens": dict(T=65535, count=65535, width=512, page=64, max_new=1),
    "the hint too small": dict(T=64 * 8192, count=64, width=128, page=64, max_new=1),
    "2^20 by 2^20 of 64 heads": dict(T=1 << 20, width=1 << 14, page=64),
    "2^31 - 1 entries": dict(T=1, heads=1, kv_heads=1, width=0x7fffffff, page=1),
}.items():
    kw = dict(dict(heads=64, kv_heads=8, dim=128), **kw)
    result[name] = attend(w=w, **kw)
""")
    for name, (st, launches) in out.items():
        tile = name not in ("2^20 by 2^20 of 64 heads", "2^31 - 1 entries")
        assert st == 0, name
        assert [x[0] for x in launches] == (["attend_tile", "weights_tile"] if tile else ["attend_any", "weights_any"]), name
        assert all(x[2] for x in launches), (name, launches)
