"""Refusals of the operators' entry points, found on the host before anything is
enqueued: no GPU is needed."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    __graft_entry__._lib_build_module().build()
    import paper_2609_37617_gb300 as p
    return p


A = 0x7000_0000_0000  # an address that is looked at and never read


def cache(lib, **kw):
    c = lib.as2d_cache(A, A + 4096, 2, 2, 4, 256, 128)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def rows(lib, counts=(5, 3), **kw):
    arr = (ctypes.c_int32 * len(counts))(*counts)
    r = lib.as2d_tree_rows(A, lib.AS2D_TYPE_BF16, 28, 28 * 128, A, 0, ctypes.addressof(arr), None, 0.1)
    r.keep = arr
    for n, v in kw.items():
        setattr(r, n, v)
    return r


def attention(lib, c=None, r=None, layer=0, out=A, ws=A, ws_bytes=1 << 40):
    c = cache(lib) if c is None else c
    r = rows(lib) if r is None else r
    return lib._lib.as2d_tree_attention(ctypes.byref(c), layer, ctypes.byref(r), out, None, ws, ws_bytes, None, None)


def weights(lib, c=None, r=None, layer=0, lse=A, w=A):
    c = cache(lib) if c is None else c
    r = rows(lib) if r is None else r
    return lib._lib.as2d_attention_weights(ctypes.byref(c), layer, ctypes.byref(r), lse, w, None, None)


BAD_CACHES = [(dict(k=None), -1), (dict(v=None), -1), (dict(k=A + 8), -1), (dict(n_layers=0), -1), (dict(batch=0), -1),
              (dict(batch=65), -1), (dict(n_kv=0), -1), (dict(capacity=0), -1), (dict(capacity=65537), -4),
              (dict(head_dim=96), -4), (dict(head_dim=0), -4)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_bad_caches(lib, change, status):
    c = cache(lib, **change)
    assert attention(lib, c) == status and lib.as2d_last_error()
    assert weights(lib, c) == status
    keep = (ctypes.c_int32 * 65)()
    assert lib._lib.as2d_cache_evict(ctypes.byref(c), A, A, keep, 0, A, 1 << 40, None) == status


BAD_ROWS = [(dict(q=None), -1), (dict(q=A + 2), -1), (dict(q_type=2), -1), (dict(n_q=0), -1), (dict(n_q=27), -1),
            (dict(n_q=4 * 2000), -4), (dict(q_stride=28 * 128 - 8), -1), (dict(q_stride=28 * 128 + 1), -1),
            (dict(kv_len=None), -1), (dict(max_len=-1), -1), (dict(max_len=257), -1), (dict(rows=None), -1),
            (dict(visible=A + 4), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1),
            (dict(scale=float("inf")), -1)]


@pytest.mark.parametrize("change,status", BAD_ROWS)
def test_bad_rows(lib, change, status):
    r = rows(lib, **change)
    if change.get("n_q") == 8000:
        r.q_stride = 8000 * 128
    assert attention(lib, r=r) == status and lib.as2d_last_error()
    assert weights(lib, r=r) == status


def test_bad_counts_and_layers(lib):
    for counts, status in (((-1, 3), -1), ((65, 1), -1), ((1, 64), 0)):
        if status:
            assert attention(lib, r=rows(lib, counts)) == status
    assert attention(lib, cache(lib, capacity=30), rows(lib, (31, 1))) == -2
    for layer in (-1, 2):
        assert attention(lib, layer=layer) == -1 and weights(lib, layer=layer) == -1
    assert lib._lib.as2d_tree_attention(None, 0, ctypes.byref(rows(lib)), A, None, A, 1 << 40, None, None) == -1
    assert lib._lib.as2d_tree_attention(ctypes.byref(cache(lib)), 0, None, A, None, A, 1 << 40, None, None) == -1


def test_bad_outputs_and_workspaces(lib):
    assert attention(lib, out=None) == -1 and attention(lib, out=A + 4) == -1
    assert attention(lib, ws=None) == -1 and attention(lib, ws=A + 128) == -1
    assert attention(lib, ws_bytes=16) == -1 and attention(lib, ws_bytes=-1) == -1
    assert weights(lib, lse=None) == -1 and weights(lib, w=None) == -1
    n = ctypes.c_int64()
    assert lib._lib.as2d_cache_evict_workspace(ctypes.byref(cache(lib)), ctypes.byref(n)) == 0
    # two bytes a place, four a head, in pieces of 256
    assert n.value == 16 * 256 * 2 + 256
    keep = (ctypes.c_int32 * 2)(5, 5)
    c = ctypes.byref(cache(lib))
    assert lib._lib.as2d_cache_evict(c, A, A, keep, 0, A, n.value - 1, None) == -1
    assert lib._lib.as2d_cache_evict(c, A, A, keep, -1, A, n.value, None) == -1
    assert lib._lib.as2d_cache_evict(c, None, A, keep, 0, A, n.value, None) == -1
    assert lib._lib.as2d_cache_evict(c, A, None, keep, 0, A, n.value, None) == -1
    assert lib._lib.as2d_cache_evict(c, A, A, None, 0, A, n.value, None) == -1
    keep[1] = -1
    assert lib._lib.as2d_cache_evict(c, A, A, keep, 0, A, n.value, None) == -1
    for f in (lib._lib.as2d_cache_evict_workspace, lib._lib.as2d_tree_attention_workspace):
        assert f(None, ctypes.byref(n)) == -1 and f(c, None) == -1


def test_no_rows_is_nothing_to_do(lib):
    r = rows(lib, (0, 0), q=None)
    assert attention(lib, r=r, out=None) == 0 and weights(lib, r=r, lse=None, w=None) == 0
    assert lib._lib.as2d_token_probs(None, 0, 5, 1.0, None, None) == 0


def test_bad_sampling(lib):
    f = lib._lib.as2d_token_probs
    for args in ((A, -1, 5, 1.0, A), (A, 1, 0, 1.0, A), (A, 1, 5, 0.0, A), (A, 1, 5, -1.0, A),
                 (A, 1, 5, float("nan"), A), (A, 1, 5, float("inf"), A), (None, 1, 5, 1.0, A), (A, 1, 5, 1.0, None),
                 (A + 2, 1, 5, 1.0, A), (A, 1, 5, 1.0, A + 1)):
        assert f(*args, None) == -1 and lib.as2d_last_error()
    f = lib._lib.as2d_accept_sampled
    k = (ctypes.c_int32 * 64)(*([2] * 64))
    good = [A, None, A, k, 2, 100, A, A, A]
    for at, bad in ((0, None), (2, None), (3, None), (4, 0), (4, 65), (5, 0), (6, None), (7, None), (8, None)):
        args = list(good)
        args[at] = bad
        assert f(*args, None) == -1, at
    for bad in (-1, 17):
        k[1] = bad
        assert f(*good, None) == -1


def test_scale_beyond_its_base_two_form(lib):
    """scale itself is finite, scale log2(e) is not: a score of 0 would be 0 inf."""
    r = rows(lib, scale=3e38)
    assert attention(lib, r=r) == -1 and "scale" in lib.as2d_last_error()
    assert weights(lib, r=r) == -1


def test_addresses_off_their_types(lib):
    """Addresses that are no multiple of their type's size are refused, argument by argument."""
    for off in (1, 2, 3):
        r = rows(lib, kv_len=A + off)
        assert attention(lib, r=r) == -1 and weights(lib, r=r) == -1 and "kv_len" in lib.as2d_last_error()
        c, r = ctypes.byref(cache(lib)), ctypes.byref(rows(lib))
        assert lib._lib.as2d_tree_attention(c, 0, r, A, A + off, A, 1 << 40, None, None) == -1
        assert lib._lib.as2d_tree_attention(c, 0, r, A, None, A, 1 << 40, A + off, None) == -1
        assert weights(lib, lse=A + off) == -1 and weights(lib, w=A + off) == -1
        assert lib._lib.as2d_attention_weights(c, 0, r, A, A, A + off, None) == -1
        keep = (ctypes.c_int32 * 2)(5, 5)
        assert lib._lib.as2d_cache_evict(c, A + off, A, keep, 0, A, 1 << 40, None) == -1
        assert lib._lib.as2d_cache_evict(c, A, A + off, keep, 0, A, 1 << 40, None) == -1
        k = (ctypes.c_int32 * 2)(2, 2)
        good = [A, A, A, k, 2, 100, A, A, A]
        for at in (0, 1, 2, 6, 7, 8):
            args = list(good)
            args[at] = A + off
            assert lib._lib.as2d_accept_sampled(*args, None) == -1, at
            assert "aligned" in lib.as2d_last_error()
