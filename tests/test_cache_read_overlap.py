"""mvk_cache_read into the memory of the cache that it reads is refused, and rows
beside or behind it are written (the library's host side; nothing is computed)."""
from tests.test_host_dispatch import host  # noqa: F811,F401

# Pools of 8 pages, 4 heads, 16 entries of 64 values; the rows of 3 tokens.
SETUP = """
def rows(data, type_, token=256, head=64): return L.MvkRows(data, type_, token, head)
def seqs(): return L.MvkSeqs(ptr(), 4, 2, 4, ptr(), ptr(), 1)
def call(cache, k, v, T=3, type_=0, **kw):
    rec.rec_reset()
    sq = seqs()
    k, v = (ref(rows(x, type_, **kw)) if x is not None else None for x in (k, v))
    st = lib.mvk_cache_read(ctypes.cast(ref(cache), ctypes.POINTER(L.MvkKv)), ref(sq), T, k, v, None)
    return [st, rec.rec_count()]
def both(cache, x, **kw): return [call(cache, x, None, **kw), call(cache, None, x, **kw), call(cache, ptr(), x, **kw)]
"""
NO, YES = [-1, 0], [0, 1]


def test_caches_of_floats(host):  # noqa: F811
    out = host(SETUP + """
K, V = ptr(), ptr()
size = 2 * 8 * 4 * 16 * 64
cache = L.MvkKv(K, V, 0, 8, 4, 16, 64, 4096, 1024, 64, 4096, 1024, 64)
row = 2 * 3 * 256
result["apart"] = both(cache, ptr())
for name, p in (("K", K), ("V", V)):
    result[name] = both(cache, p)
    result[name + ", the last value"] = both(cache, p + size - 2)
    result[name + ", behind it"] = both(cache, p + size)
    result[name + ", the first value"] = both(cache, p - row + 2)
    result[name + ", before it"] = both(cache, p - row)
result["no rows"] = call(cache, K, None, T=0)
""")
    for name, got in out.items():
        if name == "no rows":
            assert got == [0, 0]
        else:
            assert got == [YES if "apart" in name or "behind" in name or "before" in name else NO] * 3, name


def test_caches_in_8_bits(host):  # noqa: F811
    out = host(SETUP + """
K, V, kx, vx = ptr(), ptr(), ptr(), ptr()
for kind in (L.MVK_TYPE_E4M3, L.MVK_TYPE_I8):
    cache = L.MvkKv8(K, V, kind, 8, 4, 16, 64, 4096, 1024, 64, 4096, 1024, 64, kx, vx, 64, 16, 1, 64, 16, 1)
    for name, p, size in (("K", K, 32768), ("V", V, 32768), ("k_exp", kx, 512), ("v_exp", vx, 512)):
        for type_ in (0, 2):
            row = (2 if type_ == 0 else 4) * 3 * 256
            name = f"{name} {kind} {type_}"
            result[name] = both(cache, p, type_=type_)
            result[name + ", the last"] = both(cache, p + size - 4, type_=type_)
            result[name + ", behind"] = both(cache, p + size, type_=type_)
            result[name + ", the first"] = both(cache, p - row + 4, type_=type_)
            result[name + ", before"] = both(cache, p - row, type_=type_)
""")
    assert len(out) == 80
    for name, got in out.items():
        assert got == [YES if "behind" in name or "before" in name else NO] * 3, name


def test_parts_of_one_buffer(host):  # noqa: F811
    """Entries before heads, and pools that are parts of the pages of one buffer: rows in
    what they leave free are written, where the strides tell them apart."""
    out = host(SETUP + """
x = ptr()
# pages x (K, V, free) x entries x heads x dim
page = 3 * 16 * 4 * 64
cache = L.MvkKv(x, x + 2 * 4096, 0, 8, 4, 16, 64, page, 64, 256, page, 64, 256)
result["free"] = both(cache, x + 2 * 8192, token=page)
result["free, a value short"] = both(cache, x + 2 * 8192 - 2, token=page)
result["rows over the next page"] = both(cache, x + 2 * 8192 + 2 * 4096 - 2 * 254, token=page)
result["rows up to it"] = both(cache, x + 2 * 8192 + 2 * 4096 - 2 * 256, token=page)
""")
    assert out == {"free": [YES] * 3, "free, a value short": [NO] * 3, "rows over the next page": [NO] * 3,
                   "rows up to it": [YES] * 3}
