"""Refusals of the cache calls, on the CPU: arguments are checked before a device is touched.  The context is a block of
zeroed memory that begins with a configuration, which is all that the checks read."""
import ctypes as C

import pytest

from paper_2609_22098_b200 import binding

OK = 0x1000          # an aligned address that nothing reads: every call below is refused


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


@pytest.fixture()
def ctx():
    buf = (C.c_uint64 * 1024)()
    cfg = binding.TsConfig(1024, 4, 8, 4, 16, 8, 1, 1, 1, 1, 0, 0.67, -0.46, -10, 10, None)
    C.memmove(buf, C.byref(cfg), C.sizeof(cfg))
    C.cast(C.addressof(buf) + C.sizeof(cfg), C.POINTER(C.c_uint64))[1] = (1 << 32) - 1   # no device has this number
    return buf


def layout(**kw):
    d = dict(Hq=8, Hkv=2, Dh=128, page_size=16, n_pages=10, max_pages=4, dtype=1, k_exp=0, v_exp=0)
    d.update(kw)
    return binding.TsCacheLayout(*d.values())


BAD_LAYOUTS = [dict(Hq=7), dict(Hkv=0), dict(Hq=0), dict(Hq=2048), dict(Dh=96), dict(Dh=0), dict(page_size=8), dict(page_size=24), dict(page_size=8192), dict(page_size=0),
               dict(n_pages=0), dict(max_pages=0), dict(n_pages=1 << 28), dict(max_pages=1 << 28), dict(dtype=2), dict(k_exp=31), dict(v_exp=-31), dict(page_size=-16)]


def reserve(lib, ctx, lay, B=2, ptrs=None):
    p = [OK] * 10 if ptrs is None else ptrs
    return lib.ts_cache_reserve(ctx, lay and C.byref(lay), B, *p, None)


def append(lib, ctx, lay, rows=3, k=OK, ldk=256, v=OK, ldv=256, rest=None):
    return lib.ts_cache_append(ctx, lay and C.byref(lay), rows, k, ldk, v, ldv, *(rest or [OK] * 4), None)


def attention(lib, ctx, lay, B=2, q=OK, ldq=1024, ptrs=None, scale=0.1, out=OK, ldo=1024, lse=OK, ws=OK, n=1 << 40):
    return lib.ts_tree_attention(ctx, lay and C.byref(lay), B, q, ldq, *(ptrs or [OK] * 5), scale, out, ldo, lse, ws, n, None)


def commit(lib, ctx, lay, B=2, layers=3, stride=None, ptrs=None):
    stride = lib.ts_cache_bytes(C.byref(lay)) if stride is None else stride
    return lib.ts_cache_commit(ctx, C.byref(lay), B, layers, stride, *(ptrs or [OK] * 6), None)


@pytest.mark.parametrize("kw", BAD_LAYOUTS, ids=str)
def test_layouts(lib, ctx, kw):
    lay = layout(**kw)
    assert lib.ts_cache_bytes(C.byref(lay)) == 0
    assert lib.ts_tree_attention_workspace_bytes(ctx, C.byref(lay), 2) == 0
    for call in (reserve, append, attention):
        assert call(lib, ctx, lay) == -2
    assert commit(lib, ctx, lay, stride=1 << 30) == -2


def test_sizes_of_a_layer(lib):
    assert lib.ts_cache_bytes(C.byref(layout())) == 10 * 2 * 18 * 128
    assert lib.ts_cache_bytes(C.byref(layout(Dh=64, page_size=48, n_pages=7))) == 7 * 2 * 3 * 18 * 64
    assert lib.ts_cache_bytes(None) == 0
    big = layout(n_pages=1 << 26, Hkv=8)
    assert lib.ts_cache_bytes(C.byref(big)) == (1 << 26) * 8 * 18 * 128


def test_null_context_and_layout(lib, ctx):
    for call in (reserve, append, attention, commit):
        assert call(lib, None, layout()) == -1
    for call in (reserve, append, attention):
        assert call(lib, ctx, None) == -1
    assert b"null layout" in lib.ts_last_error_string()


@pytest.mark.parametrize("B", [0, -1, 9])
def test_batch(lib, ctx, B):
    assert reserve(lib, ctx, layout(), B=B) == -1 and attention(lib, ctx, layout(), B=B) == -1 and commit(lib, ctx, layout(), B=B) == -1
    assert lib.ts_tree_attention_workspace_bytes(ctx, C.byref(layout()), B) == 0


def test_pointers(lib, ctx):
    for bad in (None, OK + 2):
        for i in range(10):
            if bad is None and i == 1:
                continue   # n_nodes may be NULL
            assert reserve(lib, ctx, layout(), ptrs=[bad if j == i else OK for j in range(10)]) == -1, i
        for i in range(4):
            if bad is None and i >= 2:
                continue   # k_val, v_val may be NULL
            assert append(lib, ctx, layout(), rest=[bad if j == i else OK for j in range(4)]) == -1, i
        assert append(lib, ctx, layout(), k=bad) == -1 and append(lib, ctx, layout(), v=bad) == -1
        for i in range(5):
            if bad is None and i >= 3:
                continue   # n_nodes (without a mask) and mask may be NULL
            assert attention(lib, ctx, layout(), ptrs=[bad if j == i else OK for j in range(5)]) == -1, i
        assert attention(lib, ctx, layout(), q=bad) == -1 and attention(lib, ctx, layout(), out=bad) == -1 and attention(lib, ctx, layout(), ws=bad) == -1
        for i in range(6):
            assert commit(lib, ctx, layout(), ptrs=[bad if j == i else OK for j in range(6)]) == -1, i
    assert attention(lib, ctx, layout(), lse=OK + 1) == -1
    assert attention(lib, ctx, layout(), ptrs=[OK, OK, OK, None, OK]) == -1   # a mask without n_nodes


def test_strides_scales_and_workspace(lib, ctx):
    for ld in (255, 260, 0, -256):   # below Hkv * Dh, no multiple of eight bf16
        assert append(lib, ctx, layout(), ldk=ld) == -1 and append(lib, ctx, layout(), ldv=ld) == -1
    assert append(lib, ctx, layout(dtype=0), ldk=258) == -1
    assert append(lib, ctx, layout(), rows=-1) == -1 and append(lib, ctx, layout(), rows=0) == 0
    for ld in (1023, 1028):
        assert attention(lib, ctx, layout(), ldq=ld) == -1 and attention(lib, ctx, layout(), ldo=ld) == -1
    for s in (float("nan"), float("inf"), -float("inf")):
        assert attention(lib, ctx, layout(), scale=s) == -1
    assert commit(lib, ctx, layout(), layers=0) == -1 and commit(lib, ctx, layout(), layers=5000) == -1
    assert commit(lib, ctx, layout(), stride=16) == -1 and commit(lib, ctx, layout(), stride=10 * 2 * 18 * 128 + 8) == -1


def test_another_device_is_refused(lib, ctx):
    """All arguments are fine here; the context's device is not the current one (or there is none)."""
    assert reserve(lib, ctx, layout()) == -1
    assert b"device" in lib.ts_last_error_string()
    assert append(lib, ctx, layout()) == -1 and b"device" in lib.ts_last_error_string()
    assert commit(lib, ctx, layout()) == -1 and b"device" in lib.ts_last_error_string()


def test_scales_beyond_the_range(lib, ctx):
    """|scale| and |scale| * 2^k_exp may be 1e30 at most: their product with the queries' power of two has to be a float."""
    for scale, k_exp in ((2e30, 0), (-2e30, -30), (1e22, 30), (-1e22, 30)):
        assert attention(lib, ctx, layout(k_exp=k_exp), scale=scale) == -1 and b"scale" in lib.ts_last_error_string()
    assert attention(lib, ctx, layout(k_exp=-30), scale=1e30) == -1 and b"device" in lib.ts_last_error_string()
    assert attention(lib, ctx, layout(k_exp=30), scale=9e20) == -1 and b"device" in lib.ts_last_error_string()
