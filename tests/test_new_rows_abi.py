"""Refusals of the entry points between a projection and its attention, found on the
host before anything is enqueued: no GPU is needed."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    __graft_entry__._lib_build_module().build()
    import paper_2609_37617_gb300 as p
    return p


A = 0x7000_0000_0000  # an address that is looked at and never read


def changed(c, kw):
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def cache(lib, **kw):
    return changed(lib.as2d_cache(A, A + 4096, 2, 2, 4, 256, 128), kw)


def cache4(lib, **kw):
    return changed(lib.as2d_cache4(A, A, A, A, 2, 2, 4, 256, 128), kw)


def new_rows(lib, counts=(5, 3), **kw):
    arr = (ctypes.c_int32 * len(counts))(*counts)
    w = 36 * 128
    r = lib.as2d_new_rows(A, A, A, lib.AS2D_TYPE_BF16, 28, w, w, w, A, ctypes.addressof(arr), None, None, None,
                          1e-6, 1e6, 128)
    r.keep = arr
    return changed(r, kw)


def tree_rows(lib, counts=(5, 3), **kw):
    arr = (ctypes.c_int32 * len(counts))(*counts)
    r = lib.as2d_tree_rows(A, lib.AS2D_TYPE_BF16, 28, 28 * 128, A, 0, ctypes.addressof(arr), None, 0.1)
    r.keep = arr
    return changed(r, kw)


def append(lib, c=None, r=None, layer=0, out=A, err=None):
    """The status of both kinds of append, which refuse the same."""
    r = new_rows(lib) if r is None else r
    a = lib._lib.as2d_cache_append(ctypes.byref(cache(lib, **(c or {}))), layer, ctypes.byref(r), out, err, None)
    kw = {n: v for n, v in (c or {}).items()}
    b = lib._lib.as2d_cache4_append(ctypes.byref(cache4(lib, **kw)), layer, ctypes.byref(r), out, err, None)
    assert a == b and lib.as2d_last_error()
    return a


def attention4(lib, c=None, r=None, layer=0, out=A, lse=None, ws=A, ws_bytes=1 << 40, err=None):
    c = cache4(lib) if c is None else c
    r = tree_rows(lib) if r is None else r
    return lib._lib.as2d_cache4_attention(ctypes.byref(c), layer, ctypes.byref(r), out, lse, ws, ws_bytes, err, None)


def prompt(lib, c=None, r=None, layer=0, out=A, lse=None, ws=A, ws_bytes=1 << 40, err=None):
    c = cache(lib) if c is None else c
    r = tree_rows(lib) if r is None else r
    return lib._lib.as2d_prompt_attention(ctypes.byref(c), layer, ctypes.byref(r), out, lse, ws, ws_bytes, err, None)


def convert(lib, c4=None, c=None, layer=-1, start=None, end=A, most=0, err=None):
    c4, c = ctypes.byref(cache4(lib) if c4 is None else c4), ctypes.byref(cache(lib) if c is None else c)
    a = lib._lib.as2d_cache4_write(c4, c, layer, start, end, most, err, None)
    b = lib._lib.as2d_cache4_read(c4, c, layer, start, end, most, err, None)
    assert a == b and lib.as2d_last_error()
    return a


BAD_CACHES = [(dict(k=None), -1), (dict(v=None), -1), (dict(k=A + 8), -1), (dict(n_layers=0), -1), (dict(batch=0), -1),
              (dict(batch=65), -1), (dict(n_kv=0), -1), (dict(capacity=0), -1), (dict(capacity=65537), -4),
              (dict(head_dim=96), -4), (dict(head_dim=0), -4)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_bad_caches(lib, change, status):
    assert append(lib, change) == status
    assert attention4(lib, cache4(lib, **change)) == status and prompt(lib, cache(lib, **change)) == status
    assert convert(lib, c4=cache4(lib, **change)) == status and convert(lib, c=cache(lib, **change)) == status


def test_bad_scales(lib):
    for change in (dict(k_scale=None), dict(v_scale=None), dict(k_scale=A + 4), dict(v_scale=A + 2)):
        c = cache4(lib, **change)
        r = new_rows(lib)
        assert attention4(lib, c) == -1 and convert(lib, c4=c) == -1 and "scale" in lib.as2d_last_error()
        assert lib._lib.as2d_cache4_append(ctypes.byref(c), 0, ctypes.byref(r), A, None, None) == -1


BAD_NEW = [(dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(q=A + 8), -1), (dict(k=A + 2), -1),
           (dict(v=A + 4), -1), (dict(type=2), -1), (dict(n_q=0), -1), (dict(n_q=70000), -4),
           (dict(q_stride=28 * 128 - 8), -1), (dict(k_stride=4 * 128 - 8), -1), (dict(v_stride=4 * 128 - 8), -1),
           (dict(q_stride=36 * 128 + 4), -1), (dict(v_stride=2 ** 62), -1), (dict(kv_len=None), -1),
           (dict(kv_len=A + 2), -1), (dict(rows=None), -1), (dict(positions=A + 1), -1), (dict(q_norm=A + 4), -1),
           (dict(k_norm=A + 8), -1), (dict(q_norm=A, eps=-1.0), -1), (dict(k_norm=A, eps=float("nan")), -1),
           (dict(theta=0.0), -1), (dict(theta=float("inf")), -1), (dict(rotary=-16), -1), (dict(rotary=16), -1),
           (dict(rotary=144), -1)]


@pytest.mark.parametrize("change,status", BAD_NEW)
def test_bad_new_rows(lib, change, status):
    assert append(lib, r=new_rows(lib, **change)) == status


def test_bad_appends(lib):
    for counts, status in (((-1, 3), -1), ((257, 1), -2)):
        assert append(lib, r=new_rows(lib, counts)) == status
    assert append(lib, layer=-1) == -1 and append(lib, layer=2) == -1
    assert append(lib, out=None) == -1 and append(lib, out=A + 8) == -1 and append(lib, err=A + 2) == -1
    f, g = lib._lib.as2d_cache_append, lib._lib.as2d_cache4_append
    assert f(None, 0, ctypes.byref(new_rows(lib)), A, None, None) == -1
    assert g(None, 0, ctypes.byref(new_rows(lib)), A, None, None) == -1
    assert f(ctypes.byref(cache(lib)), 0, None, A, None, None) == -1
    none = new_rows(lib, (0, 0), q=None, k=None, v=None)
    assert f(ctypes.byref(cache(lib)), 0, ctypes.byref(none), None, None, None) == 0
    assert g(ctypes.byref(cache4(lib)), 0, ctypes.byref(none), None, None, None) == 0


def test_bad_conversions(lib):
    for change in (dict(n_layers=1), dict(batch=1), dict(n_kv=2), dict(head_dim=64)):
        assert convert(lib, c=cache(lib, **change)) == -1
    assert convert(lib, layer=-2) == -1 and convert(lib, layer=2) == -1
    assert convert(lib, end=None) == -1 and convert(lib, end=A + 1) == -1 and convert(lib, start=A + 2) == -1
    assert convert(lib, most=-1) == -1 and convert(lib, most=257) == -1 and convert(lib, err=A + 1) == -1
    assert convert(lib, c=cache(lib, capacity=100), most=101) == -1


BAD_ROWS = [(dict(q=None), -1), (dict(q=A + 2), -1), (dict(q_type=2), -1), (dict(n_q=0), -1), (dict(n_q=27), -1),
            (dict(n_q=4 * 2000), -4), (dict(q_stride=28 * 128 - 8), -1), (dict(q_stride=28 * 128 + 1), -1),
            (dict(kv_len=None), -1), (dict(kv_len=A + 1), -1), (dict(max_len=-1), -1), (dict(max_len=257), -1),
            (dict(rows=None), -1), (dict(visible=A + 4), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1),
            (dict(scale=float("nan")), -1), (dict(scale=3e38), -1)]


@pytest.mark.parametrize("change,status", BAD_ROWS)
def test_bad_rows(lib, change, status):
    r = tree_rows(lib, **change)
    if change.get("n_q") == 8000:
        r.q_stride = 8000 * 128
    assert attention4(lib, r=r) == status and lib.as2d_last_error()
    assert prompt(lib, r=r) == status and lib.as2d_last_error()


def test_bad_attention(lib):
    for f in (attention4, prompt):
        for layer in (-1, 2):
            assert f(lib, layer=layer) == -1
        assert f(lib, out=None) == -1 and f(lib, out=A + 4) == -1
        assert f(lib, lse=A + 2) == -1 and f(lib, err=A + 1) == -1
        assert f(lib, ws=None) == -1 and f(lib, ws=A + 128) == -1 and f(lib, ws_bytes=-1) == -1
        assert f(lib, r=tree_rows(lib, (-1, 3))) == -1
        assert f(lib, r=tree_rows(lib, (0, 0), q=None), out=None) == 0
    assert attention4(lib, r=tree_rows(lib, (65, 1))) == -1
    assert attention4(lib, cache4(lib, capacity=30), tree_rows(lib, (31, 1))) == -2
    assert prompt(lib, r=tree_rows(lib, (257, 1))) == -2
    assert prompt(lib, r=tree_rows(lib, q_type=lib.AS2D_TYPE_F32)) == -4
    assert prompt(lib, r=tree_rows(lib, visible=A)) == -1 and "visible" in lib.as2d_last_error()
    n = ctypes.c_int64()
    for f, c in ((lib._lib.as2d_cache4_attention_workspace, cache4(lib)), (lib._lib.as2d_prompt_attention_workspace, cache(lib))):
        assert f(None, ctypes.byref(n)) == -1 and f(ctypes.byref(c), None) == -1
