"""What is not finite among rows appended to a cache in 4 bits: flagged, and in its place alone."""
import math

import pytest
import torch

from tests import cache4_reference as ref
from tests import test_gpu_new_rows as rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_37617_gb300 as p
    return p


def append(lib, x):
    """(error bits, codes and scales of the rows' keys and values [rows][n_kv][..])."""
    c4, err = x.packed(), rows_of.ints([0])
    lib.Cache4(*c4).append(x.q, x.k, x.v, x.kv_len, x.rows, error_bits=err, **x.call)
    at = x.place.long()
    return err.item(), [c[0, x.of, :, at] for c in c4]


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("norm,rotary", [(False, 0), (False, 32), (False, 64), (True, 0), (True, 64)])
def test_append4_keys_and_values_not_finite(lib, d, dtype, value, norm, rotary):
    """Of a value, and of a key's dim that nothing turns, the codes are the formula's.  A turned dim reaches
    the one it is turned with, a norm the whole head: what they leave there is some code.  Every
    other row, head and block of 16 dims is as without it."""
    row, head, dim = 2, 1, 20
    x = rows_of.Rows((4, 2, d), [3], [5], dtype, norm, rotary, layers=1, seed=d)
    clean_err, clean = append(lib, x)
    assert clean_err == 0
    x.v[row, head, dim] = value
    err, got = append(lib, x)
    assert err == lib.AS2D_DEVERR_NOT_FINITE
    want = ref.pack(x.v.double())
    assert torch.equal(got[2], want[0]) and torch.equal(got[3], want[1])
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    x.v[row, head, dim] = 0.5
    _, clean = append(lib, x)
    x.k[row, head, dim] = value
    err, got = append(lib, x)
    assert err == lib.AS2D_DEVERR_NOT_FINITE
    assert torch.equal(got[2], clean[2]) and torch.equal(got[3], clean[3])
    if not norm and dim >= rotary:
        want = ref.pack(x.k.double())
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        return
    touched = range(d // 16) if norm else {dim // 16, (dim + rotary // 2) % rotary // 16}
    for blocks in touched:
        got[0][row, head, 8 * blocks:8 * blocks + 8] = clean[0][row, head, 8 * blocks:8 * blocks + 8]
        got[1][row, head, blocks] = clean[1][row, head, blocks]
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append4_largest_finite_values(lib, dtype):
    """Finite values beyond the largest scale saturate and are not flagged."""
    x = rows_of.Rows((4, 2, 128), [3], [5], dtype, False, 0, layers=1)
    x.v[1, 0, 40], x.k[4, 1, 3], x.k[0, 0, 100] = 3e38, -3e38, 7000.0
    err, got = append(lib, x)
    assert err == 0
    for y, codes, scales in ((x.k, *got[:2]), (x.v, *got[2:])):
        want = ref.pack(y.double())
        assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
